"""Attention over the paged cache for batches of far more rows than a GPU has places for."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import kind_of, make, query


@pytest.mark.parametrize("n", [20000, 300001])
@pytest.mark.parametrize("hq,hkv,dim,kind,page,order", [(4, 2, 64, "bf16", 16, "lnht"), (3, 1, 128, "f16", 5, "lnht"),
                                                        (8, 4, 96, "e4m3", 16, "lnth")])
def test_many_rows(hq, hkv, dim, kind, page, order, n):
    """Rows that name one of 60 sequences each, in any order; one sequence is long."""
    lengths = [0, 1, 2, 3000] + [1 + 37 * s % 150 for s in range(56)]
    c = make(lengths, hkv, dim, page, kind, order)
    base = query(len(lengths), hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(n)
    seq = torch.randint(4, len(lengths), (n,), device="cuda", generator=gen)
    for s, every in ((0, 1000), (1, 777), (2, 778), (3, 5001)):
        seq[s::every] = s
    got, got_lse = c.attend(0, base[seq], seq=seq.int())
    c.sync()
    want, want_lse, spread, reach = km.attend(c, 0, base, dim ** -0.5)
    off, off_lse = km.bounds(spread, reach, dim, kind_of(c), "f16" if kind == "f16" else "bf16")
    empty = torch.isinf(want_lse)[seq]
    assert torch.equal(torch.isneginf(got_lse), empty) and bool((got[empty] == 0).all())
    assert bool(((got.double() - want[seq]).abs() <= off[seq]).all())
    assert bool((torch.where(empty, 0.0, (got_lse.double() - want_lse[seq]).abs()) <= off_lse[seq]).all())
