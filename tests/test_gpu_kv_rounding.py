"""Keys and values written in 8 bits are their quotients by the scales, rounded once: next to ties, and for scales of any size."""
import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km

LAYERS, HEADS, DIM, TOKENS = 16, 64, 32, 16


def written(x, scale):
    """The 8-bit values [layers, tokens, heads, dim] that a cache with these scales (NumPy, [layers, heads]) holds of x."""
    s = torch.from_numpy(np.ascontiguousarray(scale)).cuda()
    c = g.KvCache.empty(LAYERS, 2, TOKENS, HEADS, DIM, 1, 2, dtype=torch.float8_e4m3fn, k_scale=s, v_scale=s)
    i32 = lambda v: torch.tensor([v], dtype=torch.int32, device="cuda")  # noqa: E731
    c.extend(i32(0), i32(TOKENS))
    c.write(0, i32(0), torch.tensor([0, TOKENS], device="cuda"), x, x)
    c.sync()
    page = int(c.table[0, 0])
    k, v = (t[:, page].double().cpu().numpy() for t in (c.k, c.v))
    assert np.array_equal(k, v, equal_nan=True)
    return k


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dtype,shift", [("bfloat16", 0), ("bfloat16", 90), ("bfloat16", -100), ("float16", 0)])
def test_quotients_next_to_ties(dtype, shift, sign):
    """Each scale is a value over a tie, up to three steps of 32 bits beside it.  Against the quotient in 64 bits: a value of at
    most 11 bits over a scale of 24 is 2^-40 of it away from a tie of 5 bits or on it, so that the rounding to 64 bits
    does not matter."""
    rng = np.random.default_rng(abs(shift) + sign + len(dtype))
    n = (LAYERS, HEADS)
    bits = 8 if dtype == "bfloat16" else 11
    value = np.ldexp(rng.integers(2 ** (bits - 1), 2 ** bits, n).astype(np.float64), rng.integers(-6, 7, n) - bits + shift)
    odd, e = 2 * rng.integers(8, 16, n) + 1, rng.integers(-9, 4, n)
    tie = np.where(rng.random(n) < 0.25, (2 * rng.integers(0, 8, n) + 1) * 2.0 ** -10, np.ldexp(odd.astype(np.float64), e - 1))
    scale = (value / tie).astype(np.float32)
    scale = sign * (scale.view(np.int32) + rng.integers(-3, 4, n).astype(np.int32)).view(np.float32)
    others = np.ldexp(rng.integers(2 ** (bits - 1), 2 ** bits, (LAYERS, TOKENS, HEADS, DIM)).astype(np.float64),
                      rng.integers(-6, 7, (LAYERS, TOKENS, HEADS, DIM)) - bits + shift) * rng.choice([-1, 1], DIM)
    half = rng.random((LAYERS, TOKENS, HEADS, DIM)) < 0.5
    x = np.where(half, value[:, None, :, None] * rng.choice([-1, 1, 0], (LAYERS, TOKENS, HEADS, DIM)), others)
    given = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    assert np.array_equal(given.double().cpu().numpy(), x)
    want = km.e4m3(x / scale.astype(np.float64)[:, None, :, None])
    assert np.array_equal(written(given, scale), want)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e-3, 1.0, 1e4, 1e25, 1e38])
def test_scales_of_any_size(dtype, size):
    """Random values of all sizes (subnormal ones, infinities and NaN among them) and scales, powers of two among those."""
    rng = np.random.default_rng(int(abs(np.log10(size))) + len(dtype))
    x = torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, (LAYERS, TOKENS, HEADS, DIM)).astype(np.int16)).view(getattr(torch, dtype))
    scale = (rng.uniform(0.3, 3, (LAYERS, HEADS)) * size * rng.choice([-1, 1], (LAYERS, HEADS))).astype(np.float32)
    scale[::4] = np.exp2(np.floor(np.log2(np.abs(scale[::4])))).astype(np.float32)
    scale[1::4] = (scale[1::4].view(np.int32) & ~0x7fff).view(np.float32)   # (few bits: quotients that are ties exactly)
    with np.errstate(all="ignore"):
        want = x.double().numpy() / scale.astype(np.float64)[:, None, :, None]
        want = np.where(np.isinf(want), np.copysign(448, want), km.e4m3(np.where(np.isinf(want), 0, want)))
    assert np.array_equal(written(x.cuda(), scale), want, equal_nan=True)


def test_many_tokens_of_many_scales():
    """Blocks of tokens enough that a thread block takes all layers' keys and values, with a scale of its own for each."""
    layers, heads, dim, tokens = 2, 48, 16, 20001
    gen = torch.Generator(device="cuda").manual_seed(3)
    scales = [torch.rand((layers, heads), device="cuda", generator=gen) * 0.05 + 0.01 for _ in "kv"]
    scales[0][0, ::5] = 0.75
    c = g.KvCache.empty(layers, 1300, 16, heads, dim, 1, 1300, dtype=torch.float8_e4m3fn, k_scale=scales[0], v_scale=scales[1])
    seq, n = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (0, tokens))
    c.extend(seq, n)
    k, v = (torch.randn((layers, tokens, heads, dim), device="cuda", generator=gen).bfloat16() for _ in "kv")
    c.write(0, seq, torch.tensor([0, tokens], device="cuda"), k, v)
    c.sync()
    pages = c.table[0, :-(-tokens // 16)].long()
    for held, given, scale in ((c.k, k, scales[0]), (c.v, v, scales[1])):
        for layer in range(layers):
            got = held[layer].contiguous().view(torch.uint8)[pages].view(held.dtype).flatten(0, 1)[:tokens].double().cpu().numpy()
            want = km.e4m3(given[layer].double().cpu().numpy() / scale[layer].double().cpu().numpy()[:, None])
            assert np.array_equal(got, want)
