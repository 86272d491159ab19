"""Attention over the paged cache where the terms of a row's sums differ by many orders of magnitude, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import make


def far(got, want, off):
    return float(((got.double() - want).abs() / off).max())


@pytest.mark.parametrize("ahead", [14, 16, 18, 22])
@pytest.mark.parametrize("kind,hq,hkv,dim,order", [("bf16", 8, 2, 64, "lnht"), ("f16", 8, 2, 64, "lnht"), ("f16", 40, 8, 128, "lnth"),
                                                   ("f16", 24, 2, 256, "lnht"), ("e4m3", 8, 2, 128, "lnht"),
                                                   ("e4m3", 16, 4, 192, "lnth"), ("e4m3", 64, 4, 96, "lnth")])
def test_a_token_far_ahead_whose_values_are_zero(kind, hq, hkv, dim, order, ahead):
    """What the other tokens bring, e^-ahead of its weight each, is all of the result.  A logit is value 0 of a key.

    The bound: kv_model's, and for f16 and 8 bits a term of its own for each token: as P reaches up to 2^12 at least for a
    warp's largest, the half step of f16 below 2^-14, 2^-25, is 2^-37 of that.  (22: the terms lose some of their bits.)"""
    lengths = [2, 16, 17, 64, 65, 200, 1000, 20000]
    c = make(lengths, hkv, dim, 16, kind, order)
    if kind == "e4m3":
        c.k_scale.fill_(1.0)
        c.v_scale.mul_(512.0)
    c.v.copy_((c.v.float().abs() * (1 if kind == "e4m3" else 512)).to(c.v.dtype))   # (results that f16 holds with all its bits)
    gen = torch.Generator(device="cuda").manual_seed(ahead)
    put = lambda x, y: x.copy_(y.expand(x.shape).to(x.dtype))  # noqa: E731
    put(c.k[..., 0], torch.randint(-3, 4, c.k.shape[:4], device="cuda", generator=gen) * 0.125)
    for s, n in enumerate(lengths):
        t = (n - 1) * (s % 3) // 2          # the first, a middle one, the last
        page = int(c.table[s, t // 16])
        put(c.k[0, page, t % 16, :, 0], torch.tensor(float(ahead), device="cuda"))  # (exact in every type)
        put(c.v[0, page, t % 16], torch.tensor(0.0, device="cuda"))
    q = torch.zeros((len(lengths), hq, dim), device="cuda", dtype=torch.float16 if kind == "f16" else torch.bfloat16)
    q[..., 0] = 1
    out, lse = c.attend(0, q, 1.0)
    c.sync()
    want, want_lse, spread, reach = km.attend(c, 0, q, 1.0)
    off, off_lse = km.bounds(spread, reach, dim, kind, "f16" if kind == "f16" else "bf16")
    if kind != "bf16":
        v = float(c.v.float().nan_to_num(0.0).max()) * (float(c.v_scale.max()) if kind == "e4m3" else 1.0)
        off = off + torch.tensor(lengths, device="cuda")[:, None, None] * 2.0 ** -37 * 2 * v
    assert far(out, want, off) <= 1
    assert far(lse, want_lse, off_lse) <= 1


@pytest.mark.parametrize("dtype,outlier,rest", [("bfloat16", 2.0 ** 20, 3.0), ("bfloat16", 2.0 ** -90, 2.0 ** -108),
                                                ("bfloat16", 2.0 ** 127, 2.0 ** 108), ("float16", 60000.0, 0.1)])
def test_one_large_value_in_a_query_beside_8_bit_keys(dtype, outlier, rest):
    """A query's value that is 2^18 times the others, where all keys are 0: the logits are the others'."""
    dim = 128
    c = make([1, 40, 3000], 2, dim, 16, "e4m3")
    c.k[..., 5].copy_(torch.zeros(c.k.shape[:4], device="cuda").to(c.k.dtype))
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = (torch.randn((3, 8, dim), device="cuda", generator=gen) * rest).to(getattr(torch, dtype))
    q[..., 5] = outlier
    scale = 0.3 / rest
    out, lse = c.attend(0, q, scale)
    c.sync()
    want, want_lse, spread, reach = km.attend(c, 0, q, scale)
    off, off_lse = km.bounds(spread, reach, dim, "e4m3", "f16" if dtype == "float16" else "bf16")
    assert far(out, want, off) <= 1
    assert far(lse, want_lse, off_lse) <= 1
