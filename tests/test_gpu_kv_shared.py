"""Attention of rows that share a prefix, read once for all of them, against the same in 64 bits; the bounds are kv_model's."""
import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    from test_gpu_kv_attend import check, query


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def shared_cache(prefixes, own, heads, dim, page, kind, order="lnht", seed=0, layers=1):
    """prefixes: tokens of each group's prefix; own: for each group, the tokens of each of its rows beyond it.  Rows take the prefix's
    whole pages together, as forks that were extended leave them.  What no sequence holds is NaN."""
    rng = np.random.default_rng(seed)
    lengths = [p + n for p, group in zip(prefixes, own) for n in group]
    most = max(max(km.ceil_div(n, page) for n in lengths), 1)
    total = sum(p // page for p in prefixes) + sum(km.ceil_div(p + n, page) - p // page for p, group in zip(prefixes, own) for n in group)
    pages = total + 5
    ids = rng.permutation(pages)[:total].tolist()
    table, refs, held = np.full((len(lengths), most), -1, np.int32), np.zeros(pages, np.int32), np.zeros((pages, page), bool)
    row = 0
    for p, group in zip(prefixes, own):
        common = [ids.pop() for _ in range(p // page)]
        for n in group:
            mine = common + [ids.pop() for _ in range(km.ceil_div(p + n, page) - p // page)]
            table[row, :len(mine)] = mine
            for e, x in enumerate(mine):
                refs[x] += 1
                held[x, :min(page, p + n - e * page)] = True
            row += 1
    k, v = km.pool(layers, pages, page, heads, dim, kind, order, seed)
    junk = torch.from_numpy(~held).cuda()
    for x in (k, v):
        x.view(torch.uint8 if kind == "e4m3" else torch.int16).masked_fill_(junk[None, :, :, None, None], {"e4m3": 0x7F, "bf16": 0x7FC0, "f16": 0x7E00}[kind])
    scale = [torch.rand((layers, heads), device="cuda") * 0.04 + 0.01 for _ in "kv"] if kind == "e4m3" else [None, None]
    return g.KvCache(k, v, torch.from_numpy(table).cuda(), i32(lengths), torch.from_numpy(refs).cuda(), *scale)


def groups_of(sizes):
    return i32(np.concatenate([[0], np.cumsum(sizes)]))


PREFIXES = [500, 0, 16, 1025, 33, 129, 2000]
OWN = [[1, 20, 300], [5, 0], [0, 0, 1, 17, 2], [3] * 20, [100], [1, 900], list(range(40))]
SIZES = [len(x) for x in OWN]


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("hq,hkv,dim", [(14, 2, 64), (8, 8, 128), (32, 8, 128), (16, 1, 256), (5, 1, 80), (24, 2, 96), (40, 2, 16), (71, 1, 64),
                                        (9, 3, 192), (130, 1, 128), (12, 4, 32), (6, 2, 240)])
def test_against_64_bits(kind, hq, hkv, dim):
    page, order = {"bf16": (16, "lnht"), "f16": (7, "lnth"), "e4m3": (32, "hnlt")}[kind]
    c = shared_cache(PREFIXES, OWN, hkv, dim, page, kind, order)
    q = query(sum(SIZES), hq, dim, torch.float16 if kind == "f16" or (kind == "e4m3" and hq % 2) else torch.bfloat16)
    got = c.attend_shared(0, q, groups_of(SIZES), least=0)
    c.sync()
    check(c, 0, q, dim ** -0.5, got)


@pytest.mark.parametrize("window", [1, 16, 64, 129, 1000, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("kind,dim", [("bf16", 64), ("e4m3", 128), ("f16", 256)])
def test_window(window, kind, dim):
    c = shared_cache(PREFIXES, OWN, 2, dim, 16, kind)
    q = query(sum(SIZES), 8, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    got = c.attend_shared(0, q, groups_of(SIZES), window=window, least=0)
    c.sync()
    check(c, 0, q, dim ** -0.5, got, window=window)


@pytest.mark.parametrize("n,prefix,hq,hkv,dim,kind,page", [(3, 40000, 14, 2, 64, "bf16", 16), (150, 3000, 8, 1, 128, "f16", 64), (33, 5000, 4, 2, 256, "bf16", 1),
                                                           (260, 700, 16, 2, 128, "e4m3", 100)])
def test_one_prefix(n, prefix, hq, hkv, dim, kind, page):
    """Long prefixes that are split over the GPU, and many rows; the same twice."""
    rng = np.random.default_rng(1)
    c = shared_cache([prefix], [rng.integers(0, 70, n).tolist()], hkv, dim, page, kind, "lnth")
    q = query(n, hq, dim, torch.float16 if kind == "f16" else torch.bfloat16)
    got, again = (c.attend_shared(0, q, groups_of([n]), least=0) for _ in "12")
    c.sync()
    check(c, 0, q, dim ** -0.5, got)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_rows_of_any_order_and_groups_that_are_wrong():
    """Whatever the groups, results are right: rows in another order, named twice, in groups that share nothing or less than others."""
    c = shared_cache(PREFIXES, OWN, 2, 64, 16, "bf16")
    n = sum(SIZES)
    rng = np.random.default_rng(2)
    for seq, groups in ((rng.permutation(n), groups_of(SIZES)), (np.arange(n), groups_of([n])), (np.arange(n), groups_of([])), (np.arange(n), i32([3, 7])),
                        (np.arange(n), groups_of([1] * n)), (np.repeat(np.arange(5), 9), groups_of([45])), (np.repeat(np.arange(n), 3), groups_of([3] * n)),
                        (np.arange(n), i32([2, 2, 9, 9, 9, 60])), (np.arange(n)[::-1].copy(), groups_of(SIZES[::-1]))):
        q = query(len(seq), 6, 64, torch.bfloat16)
        for window in (0, 300):
            got = c.attend_shared(0, q, groups, 0.2, i32(seq), window, least=0)
            c.sync()
            check(c, 0, q, 0.2, got, i32(seq), window)


def test_places():
    """Rows off 16-byte boundaries, results with gaps."""
    c = shared_cache(PREFIXES, OWN, 2, 64, 16, "bf16")
    n = sum(SIZES)
    for shift, pitch in ((0, 64), (1, 67), (4, 72)):
        room = torch.zeros((n, 9, pitch + shift), device="cuda").bfloat16()
        q = query(n, 6, 64, torch.bfloat16)
        at = room[:, 1:7, shift:shift + 64]
        at.copy_(q)
        out = torch.full((6, n, pitch + shift), 7.0, device="cuda").bfloat16().transpose(0, 1)[:, :, shift:shift + 64]
        c.attend_shared(0, at, groups_of(SIZES), 0.2, out=out, least=0)
        got = c.attend_shared(0, at, groups_of(SIZES), 0.2, least=0)
        c.sync()
        check(c, 0, q, 0.2, got)
        assert torch.equal(out, got[0])
        assert bool((out._base.transpose(0, 1)[:, :, :shift] == 7).all()) and bool((out._base.transpose(0, 1)[:, :, shift + 64:] == 7).all())


def test_what_a_row_does_not_see():
    """NaN before a row's window reaches it neither through keys nor through values, though others of its group see it."""
    c = shared_cache([640], [[1, 100, 300, 600]], 1, 64, 16, "bf16")
    c.k[0, int(c.table[0, 600 // 16]), 600 % 16] = torch.nan
    c.v[0, int(c.table[0, 600 // 16]), 600 % 16] = torch.nan
    q = query(4, 4, 64, torch.bfloat16)
    out, lse = c.attend_shared(0, q, groups_of([4]), window=200, least=0)
    c.sync()
    assert bool(torch.isnan(out[:2]).all()) and bool(torch.isfinite(out[2:]).all()) and bool(torch.isfinite(lse[2:]).all())
    a, la = c.attend(0, q, window=200)
    c.sync()
    assert torch.allclose(out[2:].float(), a[2:].float(), atol=2.0 ** -7, rtol=2.0 ** -7) and torch.allclose(lse[2:], la[2:], atol=1e-4)


def test_after_forks_and_in_graphs():
    """The calls as a node makes them: a prompt is cached, forked and extended; a step is captured and replayed over growing rows."""
    kv = g.KvCache.empty(1, 400, 16, 2, 64, 40, 64)
    gen = torch.Generator(device="cuda").manual_seed(0)
    new = lambda n: tuple(torch.randn((n, 2, 64), device="cuda", generator=gen).bfloat16() for _ in "kv")  # noqa: E731
    kv.extend(i32([0]), i32([555]))
    kv.write(0, i32([0]), torch.tensor([0, 555], device="cuda"), *new(555))
    rows = list(range(1, 34))
    kv.fork(i32([0] * 33), i32(rows), i32([555 - 2 * r for r in rows]))
    seq, one, o = i32(rows), i32([1] * 33), torch.arange(34, device="cuda")
    q = query(33, 14, 64, torch.bfloat16)
    k, v = new(33)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    kv.set_stream(s)
    out, lse = torch.empty_like(q), torch.empty((33, 14), device="cuda")
    groups = groups_of([20, 13])

    def step():
        kv.extend(seq, one)
        kv.write(0, seq, o, k, v)
        kv.attend_shared(0, q, groups, seq=seq, out=out, lse=lse, least=0)

    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    check(kv, 0, q, 0.125, (out, lse), seq)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step()
    for _ in range(20):
        graph.replay()
    torch.cuda.synchronize()
    kv.sync()
    check(kv, 0, q, 0.125, (out, lse), seq)
    assert kv.length[1:34].tolist() == [555 - 2 * r + 21 for r in rows]


@pytest.mark.parametrize("window,saved", [(0, 2 * 640 + 320), (500, 2 * 640 + 320 - 2 * 200 - 20)])
def test_groups_that_save_too_little(window, saved):
    """Rows are worked off together from as many saved bytes on as the caller names (2 and 1 times what the groups share), and by
    attend, bit for bit, below."""
    c = shared_cache([640, 320, 64], [[10, 60, 110] * 2, [200] * 5, [5]], 2, 64, 16, "bf16")   # (windows begin at 150 to 250, and at 20)
    q, groups = query(12, 6, 64, torch.bfloat16), groups_of([6, 5, 1])
    want = c.attend(0, q, window=window)
    for least, together in ((saved * 512, True), (saved * 512 + 1, False), (1, True), (0, True), (2 ** 63 - 1, False), (-1, False)):
        got = c.attend_shared(0, q, groups, window=window, least=least)
        c.sync()
        check(c, 0, q, 0.125, got, window=window)
        assert torch.equal(got[1], want[1]) != together
        assert together or torch.equal(got[0], want[0])


def test_much_that_is_saved():
    """Without a number: what only a few hundred rows on a long prefix save is worth it, and less is not."""
    c = shared_cache([4096], [[i % 50 for i in range(200)]], 8, 128, 64, "bf16")
    q = query(200, 16, 128, torch.bfloat16)
    for groups, launches in ((groups_of([200]), 4), (groups_of([2, 2]), 4)):   # (the tables may hold as much: found on the device)
        before = c.launch_count()
        got = c.attend_shared(0, q, groups)
        assert c.launch_count() - before == launches
        c.sync()
        check(c, 0, q, 128 ** -0.5, got)
    before = c.launch_count()
    got = c.attend_shared(0, q[:20], groups_of([20]))
    assert c.launch_count() - before == 2
    c.sync()
    check(c, 0, q[:20], 128 ** -0.5, got, i32(range(20)))


def test_refusals_and_errors():
    c = shared_cache([100], [[5, 6, 7]], 2, 64, 16, "bf16")
    q, groups = query(3, 4, 64, torch.bfloat16), groups_of([3])
    for args, more in (((0, q.float(), groups), {}), ((0, q, groups.long()), {}), ((0, q, groups.cpu()), {}), ((0, q, groups[:0]), {}),
                       ((0, q, groups), dict(seq=i32([0]))), ((0, q, groups), dict(out=q[:2]))):
        with pytest.raises(ValueError):
            c.attend_shared(*args, **more)
    for args, more in (((1, q, groups), {}), ((0, q[:, :3].contiguous(), groups), {}), ((0, q, groups), dict(window=-1)), ((0, query(4, 4, 64, torch.bfloat16), groups), {}),
                       ((0, q, groups), dict(out=q[:1].expand(3, 4, 64)))):
        with pytest.raises(g.P2PError) as e:
            c.attend_shared(*args, **more)
        assert e.value.code == g.P2P_E_INVAL
    lib = g._load()
    assert lib.p2p_kv_attend_shared_work(c.handle, -1, 4) == -1 and lib.p2p_kv_attend_shared_work(c.handle, 3, 0) == -1
    a = dict(seq=None, n_groups=1, groups=groups.data_ptr())
    for bad in (dict(work=None), dict(work=q.data_ptr() + 8), dict(groups=None, work=q.data_ptr()), dict(n_groups=-1, work=q.data_ptr())):
        b = {**a, **bad}
        assert lib.p2p_kv_attend_shared(c.handle, 0, 3, None, b["n_groups"], b["groups"], 0, q.data_ptr(), 256, 64, 0, 4, 0.1, 0, q.data_ptr(), 256, 64, None,
                                        b["work"]) == g.P2P_E_INVAL
    for bad in (dict(seq=i32([0, 99, 1])), dict(seq=i32([0, 1, -1])), dict(groups=i32([0, 4])), dict(groups=i32([2, 1])), dict(groups=i32([-1, 2]))):
        for least in (0, -1):
            got = c.attend_shared(0, q, bad.get("groups", groups), seq=bad.get("seq"), least=least)
            with pytest.raises(g.P2PError) as e:
                c.sync()
            assert e.value.code == g.P2P_E_DEVICE
            if "groups" in bad:   # (what is left ungrouped is right all the same)
                check(c, 0, q, 0.125, got)
            else:
                assert bool((got[0][1 if bad["seq"][1] == 99 else 2] == 0).all())
    c.table[1, 0] = 10 ** 6
    c.attend_shared(0, q, groups, least=0)
    with pytest.raises(g.P2PError):
        c.sync()
    assert c.attend_shared(0, q[:0], groups_of([]))[0].shape == (0, 4, 64)
    c.sync()
