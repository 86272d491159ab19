"""The paged key-value cache's tables and contents (extend, write, fork, trim, compact) against the model, bit for bit."""
import random

import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km


def i32(x):
    return torch.tensor([int(v) for v in x], dtype=torch.int32, device="cuda")


def i64(x):
    return torch.tensor([int(v) for v in x], dtype=torch.int64, device="cuda")


def make(layers=2, pages=60, page=4, heads=2, dim=16, n_seqs=12, max_pages=10, kind="bf16", order="lnht", seed=1):
    k, v = km.pool(layers, pages, page, heads, dim, kind, order, seed)
    scale = [None, None]
    if kind == "e4m3":
        gen = torch.Generator(device="cuda").manual_seed(seed)
        scale = [torch.rand((layers, heads), device="cuda", generator=gen) * 0.05 + 0.01 for _ in "kv"]
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    c = g.KvCache(k, v, zeros(n_seqs, max_pages), zeros(n_seqs), zeros(pages), *scale)
    return c, km.Model(c.k, c.v, c.table, c.length, c.refs, *scale)


def rows(c, tokens, kind=None, seed=0, layers=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = kind or (torch.bfloat16 if c.k.element_size() == 1 else c.k.dtype)
    return [torch.randn((layers or c.layers, tokens, c.heads, c.dim), device="cuda", generator=gen).to(dtype) for _ in "kv"]


def grow(c, m, seq, count, seed=0):
    """Extend and write both."""
    c.extend(i32(seq), i32(count))
    m.extend(seq, count)
    off = np.concatenate([[0], np.cumsum(count)])
    k, v = rows(c, int(off[-1]), seed=seed)
    c.write(0, i32(seq), i64(off), k, v)
    m.write(0, seq, off, k, v)


@pytest.mark.parametrize("kind", ["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("page,order", [(1, "lnth"), (4, "lnht"), (7, "nlth"), (16, "hlnt"), (3, "tnlh")])
def test_random_calls(kind, page, order):
    rng = random.Random(page * 10 + len(kind))
    c, m = make(layers=3, pages=90, page=page, heads=3, dim=32, n_seqs=14, max_pages=12, kind=kind, order=order, seed=page)
    for step in range(60):
        free = int((m.refs == 0).sum())
        what = rng.choice(["extend", "extend", "fork", "trim", "compact"])
        full = [s for s in range(14) if m.length[s] > 0]
        empty = [s for s in range(14) if m.length[s] == 0]
        if what == "extend":
            seq = rng.sample(range(14), rng.randint(1, 6))
            count = [rng.randint(0, min(3 * page, 12 * page - int(m.length[s]))) for s in seq]
            if sum(km.ceil_div(x, page) + 1 for x in count) > free:
                continue
            grow(c, m, seq, count, step)
        elif what == "fork" and full and empty:
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(full) for _ in dst]
            n = [rng.randint(0, int(m.length[s])) for s in src]
            c.fork(i32(src), i32(dst), i32(n))
            m.fork(src, dst, n)
        elif what == "trim" and full:
            seq = rng.sample(full, rng.randint(1, len(full)))
            to = [rng.choice([0, rng.randint(0, int(m.length[s])), int(m.length[s])]) for s in seq]
            c.trim(i32(seq), i32(to))
            m.trim(seq, to)
        elif what == "compact":
            c.compact()
            m.compact()
        if step % 5 == 0:
            m.same(c)
    c.sync()
    m.same(c)
    st = c.stats()
    used = np.nonzero(m.refs)[0]
    assert st == dict(pages_used=len(used), pages_shared=int((m.refs > 1).sum()), pages_end=int(used.max(initial=-1)) + 1,
                      tokens=int(m.length.sum()))


def test_large_tables():
    """More sequences than a CTA has threads, pages beyond one round of the scan, long and empty items side by side."""
    c, m = make(layers=1, pages=9000, page=2, heads=1, dim=16, n_seqs=3000, max_pages=4100, seed=3)
    rng = random.Random(5)
    seq = rng.sample(range(3000), 2500)
    count = [rng.choice([0, 1, 1, 2, 3]) for _ in seq]
    count[7], count[1900] = 4000, 0
    grow(c, m, seq, count)
    c.sync()
    m.same(c)
    drop = rng.sample(seq, 1200)
    c.trim(i32(drop), i32([0] * 1200))
    m.trim(drop, [0] * 1200)
    src, n = [seq[7]] * 1100, [rng.randint(1, 40) for _ in range(1100)]
    dst = [s for s in drop if s != seq[7]][:1100]
    if seq[7] in drop:
        grow(c, m, [seq[7]], [100], 9)
    c.fork(i32(src), i32(dst), i32(n))
    m.fork(src, dst, n)
    grow(c, m, dst, [1] * 1100, 4)   # many copies of shared pages
    c.compact()
    m.compact()
    c.sync()
    m.same(c)


def test_lists_longer_than_shared_memory_holds():
    """More than 8,192 items: planned in scratch by one CTA of the cluster."""
    c, m = make(layers=1, pages=40000, page=2, heads=1, dim=16, n_seqs=20000, max_pages=6, seed=4)
    rng = random.Random(6)
    rows = rng.sample(range(20000), 20000)
    first, second = rows[:9001], rows[9001:18002]
    grow(c, m, first, [rng.randint(0, 4) for _ in first])
    n = [rng.randint(0, int(m.length[s])) for s in first]
    c.fork(i32(first), i32(second), i32(n))
    m.fork(first, second, n)
    grow(c, m, second, [rng.randint(0, 2) for _ in second], 5)   # thousands of shared pages are copied
    c.sync()
    m.same(c)
    was = snapshot(c)
    for seq, count in ((second + second[:1], [1] * 9002), (second, [1] * 9000 + [99])):
        c.extend(i32(seq), i32(count))
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE and unchanged(c, was)
    to = [rng.randint(0, int(m.length[s])) for s in first]
    c.trim(i32(first), i32(to))
    m.trim(first, to)
    c.compact()
    m.compact()
    c.sync()
    m.same(c)


def test_every_page_taken_and_given_back():
    c, m = make(pages=20, page=4, n_seqs=4, max_pages=20)
    grow(c, m, [2, 0], [44, 36])          # 11 + 9 pages
    assert c.stats()["pages_used"] == 20
    c.trim(i32([2]), i32([1]))
    m.trim([2], [1])
    grow(c, m, [0, 1], [4, 36])
    c.sync()
    m.same(c)
    c.compact()
    m.compact()
    c.sync()
    m.same(c)
    c.trim(i32([0, 1, 2, 3]), i32([0] * 4))
    c.compact()
    c.sync()
    assert c.stats() == dict(pages_used=0, pages_shared=0, pages_end=0, tokens=0)


def test_both_sharers_of_a_page_extend_in_one_call():
    c, m = make(pages=12, page=4, n_seqs=4)
    grow(c, m, [0], [6])
    c.fork(i32([0, 0]), i32([1, 2]), i32([6, 5]))
    m.fork([0, 0], [1, 2], [6, 5])
    grow(c, m, [1, 0, 2], [1, 5, 2], 3)
    c.sync()
    m.same(c)
    assert int(m.refs[1]) == 0  # each has a copy of its own: the page they shared is free


@pytest.mark.parametrize("kind,given", [("bf16", "bf16"), ("f16", "f16"), ("e4m3", "bf16"), ("e4m3", "f16")])
def test_write_strides_and_layers(kind, given):
    """Rows out of a larger tensor (a projection's output with queries beside keys and values), off 16-byte boundaries,
    with gaps between sequences' rows, into a part of the layers."""
    c, m = make(layers=4, pages=40, page=8, heads=2, dim=48, kind=kind, n_seqs=5, max_pages=8)
    seq, count = [3, 0, 4], [9, 0, 17]
    c.extend(i32(seq), i32(count))
    m.extend(seq, count)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for shift, pad in ((0, 0), (1, 3), (8, 8)):
        wide = torch.randn((2, 30, 2, 2 * 48 + 2 * pad + shift), device="cuda", generator=gen).to(km.TYPES[given])
        k, v = wide[..., shift:shift + 48], wide[..., shift + 48 + pad:shift + 96 + pad]
        off = [1, 10, 10, 27]
        c.write(1, i32(seq), i64(off), k, v)
        m.write(1, seq, off, k, v)
        c.sync()
        m.same(c)
    one = wide[0, :27, :, :48]
    c.write(3, i32(seq), i64([0, 9, 9, 26]), one, one)
    m.write(3, seq, [0, 9, 9, 26], one[None], one[None])
    c.sync()
    m.same(c)


def test_rounding_to_eight_bits():
    """Ties, values below the smallest step, beyond the largest value, infinities and NaN."""
    c, _ = make(layers=1, pages=70, page=8, heads=1, dim=16, kind="e4m3", n_seqs=2, max_pages=64)
    x = np.concatenate([[0.0, -0.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 448, 464, 480, 1e5, -465],
                        np.arange(1, 64) * 2.0 ** -10, np.arange(-40, 40) * 0.5, 17 + np.arange(30) * 0.5, 256 + 8.0 * np.arange(40)])
    x = torch.tensor(np.resize(x, 512), device="cuda").to(torch.float16).view(1, 32, 1, 16)
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(0.25)
    c.extend(i32([1]), i32([32]))
    c.write(0, i32([1]), i64([0, 32]), x, x)
    c.sync()
    for got, scale in ((c.k, 1.0), (c.v, 0.25)):
        got = got[0].float().cpu().numpy().reshape(70, 8, 16)[c.table[1, :4].cpu().numpy()].reshape(-1)
        want = km.e4m3(x.double().cpu().numpy().reshape(-1) / scale)
        assert np.array_equal(got, want)
    odd = torch.tensor([float("nan"), float("inf"), -float("inf")] + [1.0] * 13, device="cuda").to(torch.bfloat16).view(1, 1, 1, 16)
    c.extend(i32([0]), i32([1]))
    c.write(0, i32([0]), i64([0, 1]), odd, odd)
    c.sync()
    got = c.k[0, int(c.table[0, 0]), 0, 0].float().cpu().numpy()
    assert np.isnan(got[0]) and got[1] == 448 and got[2] == -448 and got[3] == 1


def test_addresses_past_32_bits():
    """A pool of more than 2^32 bytes in each array: the pages at its end are written, copied, moved and read."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    pages, page, heads, dim = 20000, 16, 8, 128       # 4 layers: 2.6 GB a layer and array
    c = g.KvCache.empty(4, pages, page, heads, dim, 4, 20)
    c.refs[:pages - 8] = 1                            # (held by someone else)
    c.extend(i32([0]), i32([40]))
    k, v = rows(c, 40)
    c.write(0, i32([0]), i64([0, 40]), k, v)
    c.fork(i32([0]), i32([1]), i32([37]))
    c.extend(i32([1]), i32([2]))
    c.sync()
    t = c.table[:2, :3].tolist()
    assert t == [[pages - 8, pages - 7, pages - 6], [pages - 8, pages - 7, pages - 5]]
    flat = lambda x, s, n: x[:, c.table[s, :3].long()].flatten(1, 2)[:, :n]
    for x, y in ((c.k, k), (c.v, v)):
        assert torch.equal(flat(x, 0, 40), y) and torch.equal(flat(x, 1, 37), y[:, :37])
    c.refs[5:7] = 0                                   # two of the others leave
    c.compact()
    c.sync()
    assert c.table[:2, :3].tolist() == [[pages - 8, pages - 7, 5], [pages - 8, pages - 7, 6]]
    for x, y in ((c.k, k), (c.v, v)):
        assert torch.equal(flat(x, 0, 40), y) and torch.equal(flat(x, 1, 37), y[:, :37])


def snapshot(c):
    return [x.clone() for x in (c.k, c.v, c.table, c.length, c.refs)]


def unchanged(c, was):
    bits = lambda x: x.contiguous().view(torch.uint8)
    return all(torch.equal(bits(a), bits(b)) for a, b in zip((c.k, c.v, c.table, c.length, c.refs), was))


@pytest.mark.parametrize("call,code", [
    (lambda c: c.extend(i32([0, 12]), i32([1, 1])), "P2P_E_DEVICE"),        # a sequence out of range
    (lambda c: c.extend(i32([-1]), i32([1])), "P2P_E_DEVICE"),
    (lambda c: c.extend(i32([1, 0, 1]), i32([1, 1, 1])), "P2P_E_DEVICE"),   # named twice
    (lambda c: c.extend(i32([0]), i32([-1])), "P2P_E_DEVICE"),
    (lambda c: c.extend(i32([2]), i32([41])), "P2P_E_DEVICE"),              # more than the table's row holds
    (lambda c: c.extend(i32([2]), i32([2 ** 31 - 1])), "P2P_E_DEVICE"),
    (lambda c: c.extend(i32([2, 3, 4, 5, 6, 7]), i32([40] * 6)), "P2P_E_NOMEM"),
    (lambda c: c.trim(i32([0]), i32([12])), "P2P_E_DEVICE"),                # more than it holds
    (lambda c: c.trim(i32([0]), i32([-1])), "P2P_E_DEVICE"),
    (lambda c: c.trim(i32([0, 0]), i32([1, 2])), "P2P_E_DEVICE"),
    (lambda c: c.trim(i32([99]), i32([0])), "P2P_E_DEVICE"),
    (lambda c: c.fork(i32([0]), i32([1]), i32([3])), "P2P_E_DEVICE"),       # dst is not empty
    (lambda c: c.fork(i32([0, 0]), i32([2, 2]), i32([3, 3])), "P2P_E_DEVICE"),
    (lambda c: c.fork(i32([0]), i32([2]), i32([12])), "P2P_E_DEVICE"),
    (lambda c: c.fork(i32([12]), i32([2]), i32([0])), "P2P_E_DEVICE"),
    (lambda c: c.fork(i32([0]), i32([-7]), i32([0])), "P2P_E_DEVICE"),
])
def test_what_does_not_hold_changes_nothing(call, code):
    c, m = make(pages=50)
    grow(c, m, [0, 1], [11, 5])
    c.sync()
    was = snapshot(c)
    call(c)
    c.extend(i32([0]), i32([1]))     # nothing takes effect before the error is reported
    k, v = rows(c, 1)
    c.write(0, i32([0]), i64([0, 1]), k, v)
    c.compact()
    c.trim(i32([0]), i32([0]))
    with pytest.raises(g.P2PError) as e:
        c.sync()
    assert e.value.code == getattr(g, code)
    assert unchanged(c, was)
    c.sync()
    grow(c, m, [0, 3], [2, 2], 7)    # and then calls work again, the same sequences too
    c.sync()
    m.same(c)


def test_writes_that_do_not_hold_are_left_out():
    c, m = make(pages=50)
    grow(c, m, [0, 1], [11, 5])
    c.fork(i32([0]), i32([2]), i32([10]))
    m.fork([0], [2], [10])
    c.sync()
    was = snapshot(c)
    k, v = rows(c, 40)
    for seq, off in (([0], [0, 12]), ([0], [0, 2]), ([12], [0, 1]), ([-1], [0, 1]), ([1], [-1, 1]), ([1], [39, 41])):
        # more tokens than held, a shared page, sequences out of range, offsets out of range
        c.write(0, i32(seq), i64(off), k, v)
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE
        assert unchanged(c, was), (seq, off)
    c.write(0, i32([0, 1]), i64([3, 1, 2]), k, v)     # offsets that decrease
    with pytest.raises(g.P2PError):
        c.sync()


def test_tables_that_do_not_hold_together():
    """Page numbers out of range and reference counts that are too small are reported and never followed."""
    c, m = make(pages=50)
    grow(c, m, [0, 1], [11, 5])
    c.sync()
    c.table[1, 1] = 50
    k, v = rows(c, 1)
    c.write(0, i32([1]), i64([0, 1]), k, v)
    with pytest.raises(g.P2PError):
        c.sync()
    c.extend(i32([1]), i32([1]))
    with pytest.raises(g.P2PError):
        c.sync()
    assert int(c.length[1]) == 5
    c.trim(i32([1]), i32([0]))
    with pytest.raises(g.P2PError):
        c.sync()
    c.length[2] = 2000000
    for call in (lambda: c.extend(i32([2]), i32([1])), lambda: c.trim(i32([2]), i32([1])), lambda: c.compact()):
        call()
        with pytest.raises(g.P2PError) as e:
            c.sync()
        assert e.value.code == g.P2P_E_DEVICE
    c.length[2] = 0
    c.sync()


def test_empty_lists_and_counts():
    c, m = make()
    none = i32([])
    c.extend(none, none)
    c.trim(none, none)
    c.fork(none, none, none)
    c.compact()
    k, v = rows(c, 0)
    c.write(0, none, i64([0]), k, v)
    c.extend(i32([3]), i32([0]))
    c.trim(i32([3]), i32([0]))
    c.fork(i32([3]), i32([4]), i32([0]))
    c.write(0, i32([3]), i64([0, 0]), k, v)
    c.sync()
    m.same(c)


def test_arguments_are_checked_on_the_host():
    c, _ = make()
    k, v = rows(c, 3)
    for call in (lambda: c.extend(i32([0]), i32([1, 2])), lambda: c.extend(i64([0]), i32([1])),
                 lambda: c.write(0, i32([0]), i64([0]), k, v), lambda: c.write(0, i32([0]), i64([0, 1]), k, v[:, :2]),
                 lambda: c.write(0, i32([0]), i64([0, 1]), k[..., :8], v[..., :8])):
        with pytest.raises(ValueError):
            call()
    many = i32(range(13))
    for call in (lambda: c.extend(many, many), lambda: c.write(1, i32([0]), i64([0, 1]), k, v),
                 lambda: c.write(-1, i32([0]), i64([0, 1]), k, v),
                 lambda: c.write(0, i32([0]), i64([0, 1]), k.half(), v.half()),
                 lambda: g.p2p_kv_extend(c.handle, -1, many, many), lambda: g.p2p_kv_trim(c.handle, 1, None, many),
                 lambda: g.p2p_kv_fork(c.handle, 1, many, many, None)):
        with pytest.raises(g.P2PError) as e:
            call()
        assert e.value.code == g.P2P_E_INVAL and g.p2p_kv_last_error(c.handle)
    c.sync()


def test_calls_in_a_graph_and_on_another_stream():
    st = torch.cuda.Stream()
    k, v = km.pool(2, 60, 4, 2, 16, "bf16", "lnht", 1)
    torch.cuda.synchronize()
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    c = g.KvCache(k, v, zeros(12, 10), zeros(12), zeros(60), stream=st)
    m = km.Model(c.k, c.v, c.table, c.length, c.refs)
    with torch.cuda.stream(st):
        grow(c, m, [0, 5], [9, 3])
        c.fork(i32([0]), i32([1]), i32([7]))
        m.fork([0], [1], [7])
        seq, one, off = i32([1, 0, 5]), i32([1, 1, 1]), i64([0, 1, 2, 3])
        nk, nv = rows(c, 3, seed=8)
        c.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            c.extend(seq, one)
            c.write(0, seq, off, nk, nv)
        for _ in range(6):
            graph.replay()
            m.extend([1, 0, 5], [1, 1, 1])
            m.write(0, [1, 0, 5], [0, 1, 2, 3], nk, nv)
    c.sync()
    m.same(c)
