"""Compaction of the paged cache looks at every length and table entry before it changes anything."""
import random

import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_pages import grow, i32, make, snapshot, unchanged


def spoil_length(c, value):
    c.length[1] = value
    return lambda: c.length.__setitem__(1, 23)


def spoil_entry(c, e, page):
    was = int(c.table[1, e])
    c.table[1, e] = page
    return lambda: c.table[1].__setitem__(e, was)


# Pages of 4 tokens: sequence 0 has 0 .. 2, sequence 1 (23 tokens) 3 .. 8, sequence 2 9 .. 10; 0 leaves.  Eight are in use.
@pytest.mark.parametrize("spoil", [
    lambda c: spoil_length(c, -1), lambda c: spoil_length(c, 41), lambda c: spoil_length(c, 2 ** 31 - 1),
    lambda c: spoil_length(c, 27),             # one entry more than was ever taken: page 0, which is free
    lambda c: spoil_entry(c, 0, -1), lambda c: spoil_entry(c, 5, 60), lambda c: spoil_entry(c, 3, 2 ** 31 - 1),
    lambda c: spoil_entry(c, 2, 1),            # free, below the pages in use
    lambda c: spoil_entry(c, 4, 50),           # free, beyond them: no page that moves
], ids=["length -1", "length 41", "length 2^31 - 1", "length 27", "entry -1", "entry 60", "entry 2^31 - 1", "entry 1", "entry 50"])
def test_nothing_moves_where_the_tables_do_not_hold(spoil):
    c, m = make(pages=60)
    grow(c, m, [0, 1, 2], [11, 23, 7])
    c.trim(i32([0]), i32([0]))
    m.trim([0], [0])
    c.sync()
    mend = spoil(c)
    was = snapshot(c)
    c.compact()
    c.extend(i32([2]), i32([1]))   # nor does any later call take effect before the error is reported
    with pytest.raises(g.P2PError) as e:
        c.sync()
    assert e.value.code == g.P2P_E_DEVICE
    assert unchanged(c, was)
    mend()
    c.compact()
    m.compact()
    c.sync()
    m.same(c)


@pytest.mark.parametrize("n_seqs,max_pages,long", [(1, 5000, 4999), (3, 2049, 2049), (4000, 700, 650), (20000, 3, 3)])
def test_every_entry_is_looked_at(n_seqs, max_pages, long):
    """Few long sequences, whose entries many warps share, and many short ones: any one entry spoilt is found."""
    c, m = make(layers=1, pages=long + 3 * n_seqs + 10, page=1, heads=1, dim=16, n_seqs=n_seqs, max_pages=max_pages)
    rng = random.Random(n_seqs)
    last = n_seqs - 1
    seq = [last] + [s for s in rng.sample(range(n_seqs), min(n_seqs, 500)) if s != last]
    grow(c, m, seq, [long] + [rng.randint(1, 3) for _ in seq[1:]])
    c.sync()
    spots = [(last, e) for e in {0, 31, 32, 255, 256, 257, 2047, 2048, long - 1} if e < long] + [(seq[-1], 0)]
    for s, e in spots:
        was = int(c.table[s, e])
        c.table[s, e] = c.refs.numel() - 1    # (a free page)
        c.compact()
        with pytest.raises(g.P2PError):
            c.sync()
        c.table[s, e] = was
    drop = seq[1::2]
    if drop:
        c.trim(i32(drop), i32([0] * len(drop)))
        m.trim(drop, [0] * len(drop))
    c.compact()
    m.compact()
    c.sync()
    m.same(c)
