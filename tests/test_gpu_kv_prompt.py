"""Attention of several new tokens a sequence over the paged key-value cache against the same in 64 bits; the bounds are kv_model's."""
import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    import kv_rows_model as rm
    from test_gpu_kv_attend import make, query


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def offsets_of(counts, first=0):
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]) + first, dtype=torch.int64, device="cuda")


def type_of(kind, hq=2):
    return torch.float16 if kind == "f16" or (kind == "e4m3" and hq % 2) else torch.bfloat16


CACHED = [0, 0, 1, 15, 16, 31, 100, 5, 1000, 64, 0, 127, 128, 600]
NEW = [1, 300, 1, 1, 17, 64, 129, 0, 33, 128, 7, 1, 2, 255]
LENGTHS = [a + b for a, b in zip(CACHED, NEW)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 64), (8, 8, 128), (32, 8, 128), (16, 1, 256), (5, 1, 80), (24, 2, 96), (40, 2, 16), (71, 1, 64),
                                        (9, 3, 192), (130, 1, 128), (12, 4, 32), (6, 2, 240), (34, 2, 256), (300, 1, 64)])
def test_against_64_bits(kind, hq, hkv, dim):
    page, order = {"bf16": (16, "lnht"), "f16": (7, "lnth"), "e4m3": (32, "hnlt")}[kind]
    c = make(LENGTHS, hkv, dim, page, kind, order)
    q = query(sum(NEW), hq, dim, type_of(kind, hq))
    got = c.attend_prompt(0, q, offsets_of(NEW))
    c.sync()
    rm.check(c, 0, q, offsets_of(NEW), dim ** -0.5, got)


@pytest.mark.parametrize("page", [1, 2, 3, 8, 16, 48, 64, 100, 128, 4096])
@pytest.mark.parametrize("order", ["lnht", "lnth", "thnl"])
def test_pages(page, order):
    lengths = [1, page, page + 1, 3 * page - 1, 333, 0, 1000]
    counts = [min(n, m) for n, m in zip(lengths, [1, 2, 3, 100, 64, 0, 200])]
    c = make(lengths, 2, 64, page, "bf16", order, layers=3)
    q = query(sum(counts), 6, 64, torch.bfloat16)
    for layer in (0, 2):
        got = c.attend_prompt(layer, q, offsets_of(counts), 0.2)
        c.sync()
        rm.check(c, layer, q, offsets_of(counts), 0.2, got)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 100, 128, 129, 500, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("kind,hq,dim", [("f16", 8, 128), ("e4m3", 2, 128), ("bf16", 14, 64), ("bf16", 6, 256)])
def test_window(window, kind, hq, dim):
    c = make(LENGTHS, 2, dim, 16, kind, "lnth")
    q = query(sum(NEW), hq, dim, type_of(kind))
    got = c.attend_prompt(0, q, offsets_of(NEW), window=window)
    c.sync()
    rm.check(c, 0, q, offsets_of(NEW), dim ** -0.5, got, window=window)


@pytest.mark.parametrize("cached,new,hq,hkv,dim,kind", [([70001], [3], 14, 2, 64, "bf16"), ([30000, 5], [200, 40], 8, 1, 128, "f16"),
                                                       ([20000], [130], 6, 2, 256, "bf16"), ([33333, 0, 1], [1, 900, 1], 4, 4, 128, "e4m3"),
                                                       ([0], [2000], 7, 1, 128, "bf16")])
def test_work_that_several_ctas_share(cached, new, hq, hkv, dim, kind):
    """Few rows over long sequences, whose range is split over the GPU and joined; the same twice."""
    c = make([a + b for a, b in zip(cached, new)], hkv, dim, 16, kind)
    q = query(sum(new), hq, dim, type_of(kind))
    for window in (0, 9001):
        got = c.attend_prompt(0, q, offsets_of(new), window=window)
        again = c.attend_prompt(0, q, offsets_of(new), window=window)
        c.sync()
        rm.check(c, 0, q, offsets_of(new), dim ** -0.5, got, window=window)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("page,dim", [(1, 64), (1, 128), (7, 80), (4, 64), (100, 256), (8, 16), (2, 192), (64, 96), (3, 256)])
@pytest.mark.parametrize("kind", ["f16", "e4m3"])
def test_pages_of_every_type(page, dim, kind):
    """Pages that boxes of whole tokens fit, and others; pages inside and across steps."""
    c = make(LENGTHS, 2, dim, page, kind, "lnth")
    q = query(sum(NEW), 10, dim, torch.float16)
    got = c.attend_prompt(0, q, offsets_of(NEW))
    c.sync()
    rm.check(c, 0, q, offsets_of(NEW), dim ** -0.5, got)


@pytest.mark.parametrize("kind,dtype", [("bf16", torch.bfloat16), ("f16", torch.float16), ("e4m3", torch.bfloat16), ("e4m3", torch.float16)])
@pytest.mark.parametrize("hq", [6, 80])
def test_scales_and_signs(kind, dtype, hq):
    """Negative and zero scales, keys with negative ones, queries of very different sizes in one tile."""
    c = make(LENGTHS, 2, 64, 16, kind)
    if kind == "e4m3":
        c.k_scale[0, 0] *= -1
        c.v_scale[0, 1] *= -1
    q = query(sum(NEW), hq, 64, dtype, size=1.0)
    q[::3] *= 8
    q[1::7] *= 2.0 ** -12
    for scale in (0.125, -0.125, 0.0, 1e-30):
        got = c.attend_prompt(0, q, offsets_of(NEW), scale)
        c.sync()
        rm.check(c, 0, q, offsets_of(NEW), scale, got)


def test_as_the_call_for_one_token():
    """One new token of each sequence: attend's results, but for the order of sums."""
    lengths = [1, 2, 17, 500, 3000, 64]
    c = make(lengths, 2, 128, 16, "f16")
    q = query(len(lengths), 14, 128, torch.float16)
    a, la = c.attend(0, q)
    b, lb = c.attend_prompt(0, q, offsets_of([1] * len(lengths)))
    c.sync()
    assert torch.allclose(a.float(), b.float(), atol=2.0 ** -9, rtol=2.0 ** -9) and torch.allclose(la, lb, atol=1e-4)


def test_lists_rows_and_places():
    """Sequences in any order and twice, rows of no sequence, rows that are not on 16-byte boundaries, results with gaps."""
    c = make(LENGTHS, 2, 64, 16, "bf16")
    seq = [8, 1, 8, 13, 5]
    counts = [33, 299, 2, 255, 64]
    o = offsets_of(counts, 5)
    rows = sum(counts) + 12
    for shift, pitch in ((0, 64), (1, 67), (4, 72)):
        room = torch.empty((rows, 9, pitch + shift), device="cuda").bfloat16()
        q = query(rows, 6, 64, torch.bfloat16)
        at = room[:, 1:7, shift:shift + 64]
        at.copy_(q)
        out = torch.full((6, rows, pitch + shift), 7.0, device="cuda").bfloat16().transpose(0, 1)[:, :, shift:shift + 64]
        lse = torch.full((rows, 6), 7.0, device="cuda")
        c.attend_prompt(0, at, o, 0.2, i32(seq), 200, out, lse)
        c.sync()
        rm.check(c, 0, q, o, 0.2, (out, lse), i32(seq), 200)
        some = torch.zeros(rows, dtype=torch.bool, device="cuda")
        some[5:rows - 7] = True
        assert bool((out[~some] == 7).all()) and bool((lse[~some] == 7).all())
        assert bool((out._base.transpose(0, 1)[:, :, :shift] == 7).all()) and bool((out._base.transpose(0, 1)[:, :, shift + 64:] == 7).all())


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("f16", 128), ("bf16", 256), ("e4m3", 64)])
def test_what_a_row_does_not_see(kind, dim):
    """Infinities and NaN in later tokens' keys and values, and in those before the window, reach no other row."""
    lengths, counts = [400, 150], [260, 150]
    c = make(lengths, 2, dim, 16, kind)
    junk = {"bf16": [torch.inf, torch.nan], "f16": [-torch.inf, torch.nan], "e4m3": [torch.nan, torch.nan]}[kind]
    bad = [(0, 350, junk[0]), (0, 333, junk[1]), (1, 149, junk[1]), (0, 9, junk[1]), (0, 200, junk[0])]
    for s, t, x in bad:
        at = (0, int(c.table[s, t // 16]), t % 16)
        for a in (c.k, c.v):
            if kind == "e4m3":
                a.view(torch.uint8)[at] = 0x7F
            else:
                a[at] = x
    q = query(sum(counts), 4, dim, type_of(kind), size=0.5)
    window = 100
    got = c.attend_prompt(0, q, offsets_of(counts), window=window)
    c.sync()
    o, lse = got
    fine = torch.ones(sum(counts), dtype=torch.bool)
    for s, t, _ in bad:
        for j in range(counts[s]):
            p = lengths[s] - counts[s] + j
            if p - window < t <= p:
                fine[j + (260 if s else 0)] = False
    fine = fine.cuda()
    want, want_lse, spread, reach = rm.prompt(c, 0, q, offsets_of(counts), dim ** -0.5, None, window)
    assert bool(fine.any()) and bool(torch.isfinite(o[fine]).all()) and bool(torch.isfinite(lse[fine]).all())
    assert bool(torch.isnan(o[~fine]).any(-1).all())
    k = km.bounds(spread[fine], torch.nan_to_num(reach[fine], 0.0), dim, kind, "f16" if q.dtype == torch.float16 else "bf16")[0]
    plain = torch.isfinite(reach[fine])
    d = (o[fine].double() - want[fine]).abs()
    assert bool((d <= k)[plain].all())


@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("f16", 128), ("f16", 256)])
def test_values_that_are_infinite(kind, dim):
    """Infinite and NaN values (with finite keys) go into the rows that see them, and into no other."""
    lengths, counts = [300, 200], [300, 130]
    c = make(lengths, 1, dim, 16, kind)
    for s, t, d, x in ((0, 100, 3, torch.inf), (0, 200, 5, -torch.inf), (0, 131, 7, torch.nan), (1, 150, 0, torch.inf), (1, 20, 1, torch.inf)):
        c.v[0, int(c.table[s, t // 16]), t % 16, 0, d] = x
    q = query(sum(counts), 3, dim, type_of(kind), size=0.5)
    got = c.attend_prompt(0, q, offsets_of(counts))
    c.sync()
    want, want_lse, spread, reach = rm.prompt(c, 0, q, offsets_of(counts), dim ** -0.5)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got[0]), torch.isnan(want)) and torch.equal(got[0][torch.isinf(want)].double(), want[torch.isinf(want)])
    off = km.bounds(spread, reach, dim, kind, kind)[0]
    assert bool(((got[0].double() - want).abs() <= off)[fine].all())


def test_tokens_far_ahead():
    """Logits hundreds above the others, rising and falling along the sequence."""
    c = make([900], 1, 64, 16, "bf16")
    q = query(300, 5, 64, torch.bfloat16)
    grow = torch.linspace(0.1, 30, 900, device="cuda")
    for order in (grow, grow.flip(0)):
        for t in range(900):
            c.k[0, int(c.table[0, t // 16]), t % 16] = (order[t] * torch.ones(64, device="cuda")).bfloat16()
        got = c.attend_prompt(0, q, offsets_of([300]))
        c.sync()
        rm.check(c, 0, q, offsets_of([300]), 0.125, got)


def test_offsets_past_32_bits():
    """Queries and results whose last rows are past 2^31 values."""
    c = make([2000], 1, 64, 16, "bf16")
    n, pitch = 1500, 1 << 21
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("no room")
    room = [torch.empty(n * pitch, dtype=torch.bfloat16, device="cuda").as_strided((n, 2, 64), (pitch, 64, 1)) for _ in "qo"]
    q = query(n, 2, 64, torch.bfloat16)
    room[0].copy_(q)
    got = c.attend_prompt(0, room[0], offsets_of([n]), out=room[1])
    c.sync()
    rm.check(c, 0, q, offsets_of([n]), 0.125, got)


def test_a_layer_far_into_a_large_pool():
    """Pages past 32-bit offsets of bytes and of values."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("no room")
    k, v = (torch.zeros((1, 70000, 1, 128, 256), dtype=torch.bfloat16, device="cuda").transpose(2, 3) for _ in "kv")
    ids = [69999, 3, 65000, 69000]
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    refs = torch.zeros(70000, dtype=torch.int32, device="cuda")
    for x in (k, v):
        for p in ids:
            refs[p] = 1
            x[0, p] = torch.randn((128, 1, 256), device="cuda").bfloat16()
    c = g.KvCache(k, v, table, i32([500]), refs)
    q = query(300, 3, 256, torch.bfloat16)
    got = c.attend_prompt(0, q, offsets_of([300]))
    c.sync()
    rm.check(c, 0, q, offsets_of([300]), 256 ** -0.5, got)


def test_graphs_and_streams():
    """Captured once, replayed over other lengths and values; on a stream of its own."""
    c = make([300, 40, 900], 2, 64, 16, "bf16")
    counts = [20, 40, 130]
    q, o = query(sum(counts), 8, 64, torch.bfloat16), offsets_of(counts)
    s = torch.cuda.Stream()
    c.set_stream(s)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.attend_prompt(0, q, o, out=out, lse=lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c.attend_prompt(0, q, o, out=out, lse=lse)
        c.attend_prompt(0, q, o, window=64)   # (what it allocates is the graph's)
    for lengths in ([300, 40, 900], [20, 555 // 16 * 0 + 40, 130], [299, 41 - 1, 500]):
        torch.cuda.synchronize()
        c.length.copy_(i32(lengths))
        q.normal_()
        out.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        rm.check(c, 0, q, o, 0.125, (out, lse))
    c.sync()


def test_refusals_and_errors():
    c = make([100, 50], 2, 64, 16, "bf16")
    q = query(30, 4, 64, torch.bfloat16)
    o = offsets_of([20, 10])
    for args, more in (((0, q.float(), o), {}), ((0, q[:, :, ::2], o), {}), ((0, q.cpu(), o), {}), ((0, q, o.int()), {}), ((0, q, o.cpu()), {}),
                       ((0, q, o), dict(seq=i32([0]))), ((0, q, o), dict(seq=i32([0, 1]).long())), ((0, q, o[:0]), {}),
                       ((0, q, o), dict(out=q[:5])), ((0, q, o), dict(lse=torch.empty((30, 4), device="cuda").half()))):
        with pytest.raises(ValueError):
            c.attend_prompt(*args, **more)
    for args, more in (((1, q, o), {}), ((-1, q, o), {}), ((0, q[:, :3].contiguous(), o), {}), ((0, q, o), dict(window=-1)),
                       ((0, q, offsets_of([1] * 30)), {}), ((0, q, o), dict(out=q[:1].expand(30, 4, 64)))):
        with pytest.raises(g.P2PError) as e:
            c.attend_prompt(*args, **more)
        assert e.value.code == g.P2P_E_INVAL
    out, lse = torch.full_like(q, 7.0), torch.full((30, 4), 7.0, device="cuda")
    for seq, offsets in (([5, 1], o), ([0, -1], o), ([1, 0], offsets_of([51, 0])), ([0, 1], torch.tensor([0, 20, 31], device="cuda")),
                         ([0, 1], torch.tensor([-3, 20, 30], device="cuda")), ([0, 1], torch.tensor([0, 40, 30], device="cuda"))):
        out.fill_(7.0)
        c.attend_prompt(0, q, offsets, seq=i32(seq), out=out, lse=lse)
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE
    # A page number out of range is not followed: zeros in its place.
    c.table[0, 2] = 10 ** 6
    got = c.attend_prompt(0, q, o)
    with pytest.raises(g.P2PError):
        c.sync()
    assert bool(torch.isfinite(got[0]).all())
    assert c.attend_prompt(0, q[:0], offsets_of([0, 0]))[0].shape == (0, 4, 64)
    c.attend_prompt(0, q, offsets_of([]))
    c.sync()


@pytest.mark.parametrize("window", [0, 50])
def test_tables_that_may_hold_the_longest_sequences(window):
    """Tables for sequences of 2^31 tokens, whose work is counted in coarser steps: units that are less than one of them are not lost."""
    lengths = [1 + (37 * i) % 300 for i in range(64)]
    counts = [min(n, 5) for n in lengths]
    c = make(lengths, 8, 16, 4096, "bf16")
    table = torch.full((64, 2 ** 31 // 4096 - 1), -1, dtype=torch.int32, device="cuda")
    table[:, :c.table.shape[1]] = c.table
    wide = g.KvCache(c.k, c.v, table, c.length, c.refs)
    q = query(sum(counts), 8, 16, torch.bfloat16)
    out, lse = torch.full_like(q, 7.0), torch.full((sum(counts), 8), 7.0, device="cuda")
    wide.attend_prompt(0, q, offsets_of(counts), window=window, out=out, lse=lse)
    wide.sync()
    rm.check(c, 0, q, offsets_of(counts), 0.25, (out, lse), window=window)
