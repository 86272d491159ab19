"""Attention of one new token over the paged key-value cache against the same in 64 bits; the bounds are kv_model's."""
import math

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km


def make(lengths, heads, dim, page, kind, order="lnht", layers=1, seed=0, spare=9):
    """A cache with these lengths, its pages in random order; what no sequence holds is NaN."""
    rng = np.random.default_rng(seed)
    used = [km.ceil_div(n, page) for n in lengths]
    pages = sum(used) + spare
    ids = rng.permutation(pages)[:sum(used)].astype(np.int32)
    table = np.full((len(lengths), max(max(used), 1)), -1, np.int32)
    held = np.zeros((pages, page), bool)
    at = 0
    for s, n in enumerate(lengths):
        table[s, :used[s]] = ids[at:at + used[s]]
        for t in range(n):
            held[table[s, t // page], t % page] = True
        at += used[s]
    k, v = km.pool(layers, pages, page, heads, dim, kind, order, seed)
    junk = torch.from_numpy(~held).cuda()
    for x in (k, v):
        x.view(torch.uint8 if kind == "e4m3" else torch.int16).masked_fill_(junk[None, :, :, None, None],
                                                                            {"e4m3": 0x7F, "bf16": 0x7FC0, "f16": 0x7E00}[kind])
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[torch.from_numpy(ids).long()] = 1
    scale = [None, None]
    if kind == "e4m3":
        scale = [torch.rand((layers, heads), device="cuda") * 0.04 + 0.01 for _ in "kv"]
    return g.KvCache(k, v, torch.from_numpy(table).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), refs.cuda(), *scale)


def query(n, heads, dim, dtype, seed=5, size=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn((n, heads, dim), device="cuda", generator=gen)).to(dtype)


def kind_of(c):
    return {torch.bfloat16: "bf16", torch.float16: "f16", torch.float8_e4m3fn: "e4m3"}[c.k.dtype]


def check(c, layer, q, scale, got, seq=None, window=0):
    out, lse = got
    want, want_lse, spread, reach = km.attend(c, layer, q, scale, seq, window)
    out_kind = "f16" if q.dtype == torch.float16 else "bf16"
    off, off_lse = km.bounds(spread, reach, c.dim, kind_of(c), out_kind)
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isneginf(lse), empty)
    assert bool((out[empty] == 0).all())
    assert bool(((out.double() - want).abs() <= off).all()), float(((out.double() - want).abs() / off).max())
    d = torch.where(empty, 0.0, (lse.double() - want_lse).abs())
    assert bool((d <= off_lse).all()), float((d / off_lse).max())


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 700, 1025, 0, 2500]


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 64), (8, 8, 128), (32, 8, 128), (16, 1, 256), (5, 1, 80), (24, 2, 96), (40, 2, 16),
                                        (71, 1, 64), (9, 3, 192), (130, 1, 128), (12, 4, 32), (6, 2, 240), (34, 2, 256)])
def test_against_64_bits(kind, hq, hkv, dim):
    page, order = {"bf16": (16, "lnht"), "f16": (7, "lnth"), "e4m3": (32, "hnlt")}[kind]
    c = make(LENGTHS, hkv, dim, page, kind, order)
    q = query(len(LENGTHS), hq, dim, torch.float16 if kind == "f16" or hq % 2 else torch.bfloat16)
    if kind == "bf16":
        q = q.bfloat16()
    got = c.attend(0, q)
    c.sync()
    check(c, 0, q, dim ** -0.5, got)


@pytest.mark.parametrize("page", [1, 2, 3, 8, 16, 48, 64, 100, 128, 4096])
@pytest.mark.parametrize("order", ["lnht", "lnth", "thnl"])
def test_pages(page, order):
    lengths = [1, page, page + 1, 3 * page - 1, 333, 0, 1000]
    c = make(lengths, 2, 64, page, "bf16", order, layers=3)
    q = query(len(lengths), 6, 64, torch.bfloat16)
    for layer in (0, 2):
        got = c.attend(layer, q, 0.2)
        c.sync()
        check(c, layer, q, 0.2, got)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100, 1000, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("kind", ["f16", "e4m3"])
def test_window(window, kind):
    c = make(LENGTHS, 2, 128, 16, kind, "lnth")
    q = query(len(LENGTHS), 8, 128, torch.float16)
    got = c.attend(0, q, window=window)
    c.sync()
    check(c, 0, q, 128 ** -0.5, got, window=window)


@pytest.mark.parametrize("n,hq,hkv,dim,kind", [(1, 32, 8, 128, "bf16"), (1, 14, 2, 64, "bf16"), (2, 7, 1, 128, "e4m3"), (3, 3, 1, 256, "f16"),
                                               (1, 48, 1, 64, "f16")])
def test_long_sequences(n, hq, hkv, dim, kind):
    """Few sequences whose length is split over the GPU and joined."""
    lengths = [70001, 3, 33333][:n]
    c = make(lengths, hkv, dim, 16, kind)
    q = query(n, hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    for _ in range(3):
        got = c.attend(0, q)
        again = c.attend(0, q)
        c.sync()
        check(c, 0, q, dim ** -0.5, got)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])   # the same sums in the same order


@pytest.mark.parametrize("hq,hkv,dim,kind,page", [(28, 4, 64, "bf16", 16), (64, 4, 80, "f16", 5), (96, 8, 64, "e4m3", 32),
                                                  (6, 2, 96, "bf16", 1), (48, 4, 192, "e4m3", 16), (12, 12, 80, "bf16", 16)])
def test_long_sequences_heads_inside_tokens(hq, hkv, dim, kind, page):
    """The same where a token's heads lie together, with and without a window that starts inside a tile."""
    lengths = [40003, 0, 9, 12345]
    c = make(lengths, hkv, dim, page, kind, "lnth")
    q = query(4, hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    for window in (0, 9001):
        got = c.attend(0, q, window=window)
        again = c.attend(0, q, window=window)
        c.sync()
        check(c, 0, q, dim ** -0.5, got, window=window)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_one_kv_head_and_many_parts(kind):
    """One row of units over the whole GPU, whose parts are joined in two steps."""
    c = make([150000], 1, 128, 16, kind)
    q = query(1, 16, 128, torch.bfloat16)
    got = c.attend(0, q)
    c.sync()
    check(c, 0, q, 128 ** -0.5, got)


@pytest.mark.parametrize("n", [1, 2, 3, 150, 400, 1300])
def test_many_sequences(n):
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(700), n))]
    lengths[n // 2] = 3000
    c = make(lengths, 2, 64, 16, "bf16")
    q = query(n, 14, 64, torch.bfloat16)
    got = c.attend(0, q)
    c.sync()
    check(c, 0, q, 0.125, got)


@pytest.mark.parametrize("hq,hkv,dim,kind,page", [(8, 4, 80, "f16", 16), (4, 2, 64, "bf16", 5), (24, 4, 64, "e4m3", 32),
                                                  (72, 4, 96, "bf16", 16), (6, 6, 192, "f16", 1), (48, 4, 176, "e4m3", 16),
                                                  (36, 2, 240, "bf16", 16), (16, 8, 48, "e4m3", 3)])
def test_many_sequences_heads_inside_tokens(hq, hkv, dim, kind, page):
    """Enough of them that a CTA takes neighbouring heads together, and one so long that many CTAs share each of its heads."""
    n = 2000
    rng = np.random.default_rng(dim)
    lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(300), n))]
    lengths[7], lengths[8], lengths[n // 2], lengths[n - 1] = 0, 3000, 40001, 0
    c = make(lengths, hkv, dim, page, kind, "lnth")
    q = query(n, hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    for window in (0, 30001):
        got = c.attend(0, q, window=window)
        again = c.attend(0, q, window=window)
        c.sync()
        check(c, 0, q, dim ** -0.5, got, window=window)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("hq,hkv,dim,kind,page", [(32, 8, 128, "bf16", 16), (28, 4, 64, "f16", 5), (64, 8, 128, "e4m3", 32),
                                                  (80, 4, 128, "bf16", 48), (6, 6, 256, "f16", 1), (48, 4, 192, "e4m3", 16)])
def test_many_short_sequences(hq, hkv, dim, kind, page):
    """Heads apart: a CTA takes neighbouring ones together for short sequences, one among them long; half of them once more
    in another order, where the long one has more weight."""
    n = 2000
    rng = np.random.default_rng(dim + hq)
    lengths = [int(x) for x in np.exp(rng.uniform(0, np.log(200), n))]
    lengths[7], lengths[8], lengths[n // 2], lengths[n - 1] = 0, 3000, 40001, 0
    c = make(lengths, hkv, dim, page, kind, "lnht")
    dtype = torch.float16 if kind == "f16" else torch.bfloat16
    got = c.attend(0, q := query(n, hq, dim, dtype))
    again = c.attend(0, q)
    c.sync()
    check(c, 0, q, dim ** -0.5, got)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    seq = torch.from_numpy(rng.permutation(n)[:n // 2].astype(np.int32)).cuda()
    got = c.attend(0, q := query(n // 2, hq, dim, dtype, 6), seq=seq)
    c.sync()
    check(c, 0, q, dim ** -0.5, got, seq)


def test_sequences_in_any_order_and_again():
    c = make(LENGTHS, 2, 64, 16, "bf16")
    seq = torch.tensor([20, 3, 3, 0, 17, 20, 5] * 7, dtype=torch.int32, device="cuda")   # (more rows than sequences)
    q = query(len(seq), 14, 64, torch.bfloat16)
    got = c.attend(0, q, seq=seq)
    c.sync()
    check(c, 0, q, 0.125, got, seq)


def test_strides_of_q_and_out():
    c = make([33, 0, 500], 2, 80, 16, "bf16")
    wide = query(3, 9, 90, torch.bfloat16)
    q = wide[:, 1:7, 5:85]                       # heads and values from the middle: no 16-byte boundaries
    room = torch.full((3, 7, 91), 7.0, device="cuda", dtype=torch.bfloat16)
    out = room[:, :6, 3:83]
    got = c.attend(0, q, out=out)
    c.sync()
    check(c, 0, q.contiguous(), 80 ** -0.5, got)
    mask = torch.ones_like(room, dtype=torch.bool)
    mask[:, :6, 3:83] = False
    assert bool((room[mask] == 7).all())
    heads_first = query(6, 3, 80, torch.bfloat16).transpose(0, 1)
    out = torch.empty((6, 3, 80), device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    got = c.attend(0, heads_first, out=out)
    c.sync()
    check(c, 0, heads_first.contiguous(), 80 ** -0.5, got)


def test_without_lse():
    c = make([33, 0, 5000], 2, 64, 16, "bf16")
    q = query(3, 14, 64, torch.bfloat16)
    out, _ = c.attend(0, q)
    again = torch.empty_like(out)
    g.p2p_kv_attend(c.handle, 0, 3, None, q.data_ptr(), 14 * 64, 64, g.P2P_KV_BF16, 14, 0.125, 0, again.data_ptr(), 14 * 64, 64, None)
    c.sync()
    assert torch.equal(out, again)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0, 8.0])
def test_scales(scale):
    c = make([1, 40, 900], 2, 64, 16, "f16")
    q = query(3, 4, 64, torch.float16)
    got = c.attend(0, q, scale)
    c.sync()
    check(c, 0, q, scale, got)


@pytest.mark.parametrize("kind,size", [("bf16", 1e30), ("bf16", 1e-30), ("e4m3", 1e6), ("e4m3", 1e-6), ("f16", 60000.0)])
def test_large_and_small_queries(kind, size):
    """Values that another type or an early product would not hold; the scale makes up for them."""
    c = make([7, 300], 2, 64, 16, kind)
    q = query(2, 14, 64, torch.float16 if kind == "f16" else torch.bfloat16, size=size / 4)
    scale = 0.5 / size
    got = c.attend(0, q, scale)
    c.sync()
    check(c, 0, q, scale, got)


def test_infinite_and_nan_values():
    """They go where the formula takes them, to the rows and values that read them alone."""
    c = make([40, 40, 40, 40], 1, 64, 16, "bf16")
    p = c.table.tolist()
    c.v[0, p[1][1], 3, 0, 5] = math.inf
    c.v[0, p[2][0], 0, 0, 9] = math.nan
    c.k[0, p[3][0], 2, 0, 0] = math.nan
    q = query(4, 2, 64, torch.bfloat16)
    out, lse = c.attend(0, q)
    c.sync()
    assert bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(lse[:3]).all())
    assert bool(torch.isposinf(out[1, :, 5]).all()) and bool(torch.isfinite(out[1, :, 6:]).all())
    assert bool(torch.isnan(out[2, :, 9]).all()) and bool(torch.isfinite(out[2, :, :9]).all())
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(lse[3]).all())
    # A key that takes a token out: its logit is -infinity.
    c = make([40], 1, 64, 16, "bf16")
    q = torch.ones((1, 2, 64), device="cuda", dtype=torch.bfloat16)
    for t in (0, 17, 39):
        c.k[0, int(c.table[0, t // 16]), t % 16, 0, 3] = -math.inf
        c.v[0, int(c.table[0, t // 16]), t % 16] = 1000.0
    out, lse = c.attend(0, q)
    c.sync()
    assert bool(torch.isfinite(out).all()) and float(out.abs().max()) < 10 and bool(torch.isfinite(lse).all())


def test_refusals():
    c = make([40, 3], 2, 64, 16, "bf16", layers=2)
    q = query(2, 4, 64, torch.bfloat16)
    for call in (lambda: c.attend(2, q), lambda: c.attend(-1, q), lambda: c.attend(0, query(2, 5, 64, torch.bfloat16)),
                 lambda: c.attend(0, q.half()), lambda: c.attend(0, q, window=-1), lambda: c.attend(0, query(3, 4, 64, torch.bfloat16))):
        with pytest.raises(g.P2PError) as e:
            call()
        assert e.value.code == g.P2P_E_INVAL
    for call in (lambda: c.attend(0, query(2, 4, 80, torch.bfloat16)), lambda: c.attend(0, q.float()),
                 lambda: c.attend(0, q, seq=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: c.attend(0, q, out=torch.empty((2, 4, 65), dtype=q.dtype, device="cuda")), lambda: c.attend(0, q.cpu())):
        with pytest.raises(ValueError):
            call()
    out, lse = c.attend(0, q[:0])
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    c.sync()


def test_what_the_device_refuses():
    """Sequences, lengths and pages out of range are reported; the other rows are what they were."""
    c = make([40, 300, 3], 2, 64, 16, "bf16")
    q = query(3, 4, 64, torch.bfloat16)
    good, good_lse = c.attend(0, q)
    c.sync()
    seq = torch.tensor([0, 3, 2], dtype=torch.int32, device="cuda")
    out, lse = c.attend(0, q, seq=seq)
    with pytest.raises(g.P2PError) as e:
        c.sync()
    assert e.value.code == g.P2P_E_DEVICE
    assert torch.equal(out[[0, 2]], good[[0, 2]]) and bool((out[1] == 0).all()) and bool(torch.isneginf(lse[1]).all())
    c.length[1] = 10 ** 6
    out, lse = c.attend(0, q)
    with pytest.raises(g.P2PError):
        c.sync()
    assert torch.equal(out[[0, 2]], good[[0, 2]]) and bool((out[1] == 0).all())
    c.length[1] = 300
    for page in (-1, 10 ** 6):
        c.table[1, 7] = page
        out, lse = c.attend(0, q)
        with pytest.raises(g.P2PError):
            c.sync()
        assert torch.equal(out[[0, 2]], good[[0, 2]])
    c.sync()


def test_graph_and_other_stream():
    c = make([100, 9000, 5], 2, 64, 16, "bf16")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    d = g.KvCache(c.k, c.v, c.table, c.length, c.refs, stream=st)
    with torch.cuda.stream(st):
        q = query(3, 14, 64, torch.bfloat16)
        out, lse = d.attend(0, q)
        st.synchronize()
        want = out.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            d.attend(0, q, out=out, lse=lse)
        for _ in range(3):
            out.zero_()
            graph.replay()
            st.synchronize()
            assert torch.equal(out, want)
        d.length.fill_(4)
        graph.replay()
        d.sync()
    check(d, 0, q, 0.125, (out, lse))
