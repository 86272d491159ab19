"""Norms, rotary positions and the write into the paged cache in one pass, against the same in 64 bits.

Bounds: a value is made of two products in 32 bits of factors that are each off by at most this much of themselves: the
normed value by (dim / 2 + 4) * 2^-24 (a sum of dim squares, a mean, a root, a quotient, two products), cosine and sine by pi * 2^-24
for the angle's rounding to 32 bits (a half turn at most) and 2^-22 for the functions, and the products and their sum by 2^-23:
(dim / 2 + 16) * 2^-24 of |a| + |b| covers them.  The result is rounded once, to its type."""
import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    import kv_rows_model as rm
    from test_gpu_kv_attend import make

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def offsets_of(counts, first=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + first, dtype=torch.int64, device="cuda")


def fused(tokens, hq, hkv, dim, dtype, seed=3):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (2 * torch.randn((tokens, hq + 2 * hkv, dim), device="cuda", generator=gen)).to(dtype).split([hq, hkv, hkv], 1)


def close(got, want, reach, dim, what):
    off = UNIT[got.dtype] * want.abs() + (dim / 2 + 16) * 2.0 ** -24 * reach * (1 + UNIT[got.dtype]) + LEAST[got.dtype]
    d = (got.double() - want).abs()
    assert bool((d <= off).all()), (what, float((d / off).max()))


def check(c, layer, seq, counts, q, k, v, rope, q_weight, k_weight, eps, first=0, out=None):
    length, page = c.length.tolist(), c.k.shape[2]
    table = c.table.tolist()
    before = [x.clone() for x in (c.k.view(torch.uint8 if c.k.element_size() == 1 else c.k.dtype), c.v.view(torch.uint8 if c.v.element_size() == 1 else c.v.dtype))]
    was = (q.clone(), k.clone(), v.clone())
    got = c.write_rotated(layer, i32(seq), offsets_of(counts, first), q, k, v, rope, q_weight, k_weight, eps, out)
    c.sync()
    q, k, v = was
    rows, pages, slots, pos = [], [], [], []
    for i, s in enumerate(seq):
        for j in range(counts[i]):
            t = length[s] - counts[i] + j
            rows.append(first + sum(counts[:i]) + j)
            pages.append(table[s][t // page])
            slots.append(t % page)
            pos.append(t)
    rows, pages, slots, pos = (torch.tensor(x, device="cuda") for x in (rows, pages, slots, pos))
    want, reach = rm.rotated(q[rows], pos, rope.radians, rope.amplitude, rope.interleaved, q_weight, eps)
    close(got[rows], want, reach, c.dim, "q")
    want, reach = rm.rotated(k[rows], pos, rope.radians, rope.amplitude, rope.interleaved, k_weight, eps)
    at = lambda x: (x[layer].view(torch.uint8)[pages, slots].view(x.dtype) if x.element_size() == 1 else x[layer][pages, slots])  # noqa: E731
    if c.k_scale is None:
        close(at(c.k), want, reach, c.dim, "k")
        assert torch.equal(at(c.v).view(torch.int16), v[rows].view(torch.int16))
    else:
        scale = c.k_scale[layer].double()[:, None]
        want, reach = want / scale, reach / scale
        stored = at(c.k).double()
        far = (stored - want.clamp(-448, 448)).abs()
        off = 2.0 ** -4 * want.abs() + 2.0 ** -10 + 2 * (c.dim / 2 + 16) * 2.0 ** -24 * reach
        assert bool((far <= off).all()), float((far / off).max())
        exact = km.e4m3((v[rows].double() / c.v_scale[layer].double()[:, None]).cpu().numpy())
        assert np.array_equal(at(c.v).double().cpu().numpy(), exact)
    # nothing else is written
    for x, b in ((c.k, before[0]), (c.v, before[1])):
        y = x.view(b.dtype).clone()
        y[layer, pages, slots] = b[layer, pages, slots]
        assert torch.equal(y.view(torch.uint8 if y.element_size() == 1 else torch.int16), b.view(torch.uint8 if b.element_size() == 1 else torch.int16))
    return got


LENGTHS = [40, 1, 130, 17, 64, 333, 5, 1000]
COUNTS = [1, 1, 100, 17, 0, 33, 2, 64]
SEQ = [3, 1, 7, 0, 5, 2, 6, 4]


def counts_for(seq):
    return [min(COUNTS[s], LENGTHS[s]) for s in seq]


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("hq,hkv,dim,rot", [(14, 2, 64, 64), (8, 8, 128, 128), (16, 1, 256, 64), (5, 1, 80, 40), (24, 2, 96, 48), (3, 1, 16, 2),
                                            (12, 4, 32, 0), (9, 3, 192, 192), (6, 2, 240, 100), (2, 2, 112, 112), (1, 1, 80, 16)])
def test_against_64_bits(kind, pairs, hq, hkv, dim, rot):
    page, order = {"bf16": (16, "lnht"), "f16": (7, "lnth"), "e4m3": (32, "hnlt")}[kind]
    c = make(LENGTHS, hkv, dim, page, kind, order, layers=2)
    dtype = torch.float16 if kind == "f16" or (kind == "e4m3" and hq % 2) else torch.bfloat16
    counts = counts_for(SEQ)
    q, k, v = fused(sum(counts), hq, hkv, dim, dtype)
    w = torch.rand((2, dim), device="cuda") + 0.5
    check(c, 1, SEQ, counts, q, k, v, g.Rope(rot, interleaved=pairs), w[0], w[1], 1e-6)
    check(c, 0, SEQ, counts, q, k, v, g.Rope(rot, theta=500.0, interleaved=pairs, amplitude=1.25), None, None, 0.0)


@pytest.mark.parametrize("dim", [8, 24, 40, 136, 248])
def test_head_sizes_of_odd_pieces(dim):
    c = make(LENGTHS, 2, dim, 16, "bf16")
    counts = counts_for(SEQ)
    for pairs, rot in ((False, dim // 16 * 16), (True, dim), (False, dim), (True, 6)):
        q, k, v = fused(sum(counts), 6, 2, dim, torch.bfloat16)
        check(c, 0, SEQ, counts, q, k, v, g.Rope(rot, interleaved=pairs), torch.rand(dim, device="cuda") + 0.5, None, 1e-5)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_rows_anywhere(kind):
    """Rows off 16-byte boundaries, gaps between them, results in place, rows of no sequence."""
    c = make(LENGTHS, 2, 64, 16, kind)
    counts = counts_for(SEQ)
    tokens = sum(counts) + 9
    gen = torch.Generator(device="cuda").manual_seed(1)
    for shift, pitch in ((0, 64), (1, 67), (8, 72)):
        room = torch.randn((tokens, 10, pitch + shift), device="cuda", generator=gen).bfloat16()[:, :, shift:shift + 64]
        q, k, v = room.split([6, 2, 2], 1)
        was = q.clone()
        got = check(c, 0, SEQ, counts, q, k, v, g.Rope(64), torch.rand(64, device="cuda"), torch.rand(64, device="cuda"), 1e-6, first=4, out=q)
        assert got is q and torch.equal(q[:4], was[:4]) and torch.equal(q[tokens - 5:], was[tokens - 5:])


def test_many_tokens_and_far_positions():
    """Enough tokens for the larger blocks, and positions whose angles 32 bits do not hold."""
    lengths = [200000, 9000, 12, 131072]
    c = make(lengths, 1, 32, 16, "bf16", spare=1)
    counts = [3000, 8000, 12, 2001]
    for pairs in (False, True):
        q, k, v = fused(sum(counts), 2, 1, 32, torch.bfloat16)
        check(c, 0, [0, 1, 2, 3], counts, q, k, v, g.Rope(32, interleaved=pairs), None, torch.rand(32, device="cuda"), 1e-6)


def test_scaled_positions():
    c = make([70000, 100], 2, 64, 16, "f16")
    q, k, v = fused(150, 4, 2, 64, torch.float16)
    for rope in (g.Rope(64, scaling="linear", factor=8.0), g.Rope(32, scaling="ntk", factor=4.0), g.Rope(64, scaling="by_parts", factor=8.0, original=4096),
                 g.Rope(64, scaling="yarn", factor=16.0, original=4096, interleaved=True), g.Rope(64, radians=np.linspace(0, 6.28, 32))):
        check(c, 0, [1, 0], [60, 90], q, k, v, rope, None, None, 1e-6)


def test_infinities_stay_in_their_pairs():
    c = make([8], 1, 64, 16, "bf16")
    q, k, v = (x.clone() for x in fused(8, 1, 1, 64, torch.bfloat16))
    q[3, 0, 5], k[4, 0, 60] = torch.inf, torch.nan
    got = c.write_rotated(0, i32([0]), offsets_of([8]), q, k, v, g.Rope(32))
    c.sync()
    bad = ~torch.isfinite(got)
    assert set(map(tuple, bad.nonzero().tolist())) == {(3, 0, 5), (3, 0, 21)}
    keys = c.k[0, c.table[0, 0], :8]
    assert (~torch.isfinite(keys)).nonzero().tolist() == [[4, 0, 60]] and torch.equal(keys[4, 0, 32:60], k[4, 0, 32:60])


def test_refusals_and_errors():
    c = make(LENGTHS, 2, 64, 16, "bf16")
    q, k, v = fused(10, 4, 2, 64, torch.bfloat16)
    rope, one = g.Rope(64), i32([0])
    o = offsets_of([10])
    for args in ((0, one, o, q.half(), k, v, rope), (0, one, o, q[:9], k, v, rope), (0, one, o, q, k[:, :1], v, rope), (0, one, o, q, k, v[:, :, ::2], rope),
                 (0, one.long(), o, q, k, v, rope), (0, one, o.int(), q, k, v, rope), (0, one, o, q.cpu(), k, v, rope),
                 (0, one, o, q, k, v, rope, torch.ones(63, device="cuda")), (0, one, o, q, k, v, rope, torch.ones(64, device="cuda").double()),
                 (0, one, o, q, k, v, rope, None, None, 1e-6, torch.empty((10, 3, 64), device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            c.write_rotated(*args)
    for args in ((1, one, o, q, k, v, rope), (-1, one, o, q, k, v, rope), (0, one, o, q, k, v, g.Rope(66)),
                 (0, one, o, q, k, v, rope, None, None, 1e-6, torch.empty((1, 4, 64), device="cuda").bfloat16().expand(10, 4, 64))):
        with pytest.raises(g.P2PError) as e:
            c.write_rotated(*args)
        assert e.value.code == g.P2P_E_INVAL
    # What the device finds: tokens are left out, their queries too, and it is reported.
    c.refs[c.table[2, 0].long()] = 2
    for seq, counts in (([99], [10]), ([-1], [10]), ([1], [10]), ([2], [10])):
        c.length[2] = 10
        out = torch.full_like(q, 7.0)
        held = c.k.clone()
        c.write_rotated(0, i32(seq), offsets_of(counts), q, k, v, rope, out=out)
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE
        assert bool((out == 7).all()) and torch.equal(c.k.view(torch.int16), held.view(torch.int16))
    c.write_rotated(0, i32([0, 3]), torch.tensor([0, 12, 6], device="cuda"), q, k, v, rope)
    with pytest.raises(g.P2PError):
        c.sync()
    c.write_rotated(0, i32([0]), o, q, k, v, rope)
    c.write_rotated(0, i32([]), offsets_of([]), q[:0], k[:0], v[:0], rope)
    c.sync()
