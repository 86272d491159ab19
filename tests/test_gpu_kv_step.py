"""A layer's calls as a node makes them, one after another: prompts that hit a cached prefix are rotated and written, attend over it and
themselves, and are then decoded a token at a time, over the prefix together.  Everything is recomputed from the tokens alone."""
import numpy as np
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import kv_model as km
    import kv_rows_model as rm


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


class Plain:
    """The projections of every token of each sequence, and attention over them in 64 bits."""

    def __init__(self, rope, q_weight, k_weight):
        self.rope, self.q_weight, self.k_weight, self.rows = rope, q_weight, k_weight, {}

    def add(self, s, q, k, v):
        old = self.rows.get(s)
        self.rows[s] = (q, k, v) if old is None else tuple(torch.cat([a, b]) for a, b in zip(old, (q, k, v)))

    def fork(self, src, dst, n):
        self.rows[dst] = tuple(x[:n] for x in self.rows[src])

    def attend(self, s, last, scale):
        """The last tokens of sequence s, each up to itself: [last, heads, dim], and sum p |v|."""
        q, k, v = self.rows[s]
        pos = torch.arange(len(q), device=q.device)
        turn = lambda x, w: rm.rotated(x, pos, self.rope.radians, self.rope.amplitude, self.rope.interleaved, w)[0]  # noqa: E731
        q, k, v = turn(q, self.q_weight), turn(k, self.k_weight), v.double()
        group = q.shape[1] // k.shape[1]
        k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
        x = scale * torch.einsum("qhd,khd->hqk", q[-last:], k)
        x = x.masked_fill(pos[None, None, :] > pos[-last:, None], -torch.inf)
        p = torch.softmax(x, -1)
        reach = scale * torch.einsum("qhd,khd->hqk", q[-last:].abs(), k.abs()).amax(-1).T
        return torch.einsum("hqk,khd->qhd", p, v), torch.einsum("hqk,khd->qhd", p, v.abs()), reach


@pytest.mark.parametrize("kind,hq,hkv,dim,pairs", [("bf16", 14, 2, 64, False), ("f16", 8, 8, 128, True), ("e4m3", 16, 2, 128, False)])
def test_prompts_then_steps(kind, hq, hkv, dim, pairs):
    dtype = torch.float16 if kind == "f16" else torch.bfloat16
    scales = [torch.full((1, hkv), 0.03, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
    kv = g.KvCache.empty(1, 300, 16, hkv, dim, 12, 64, dtype=km.TYPES[kind], k_scale=scales[0], v_scale=scales[1])
    gen = torch.Generator(device="cuda").manual_seed(1)
    rope = g.Rope(dim, interleaved=pairs, scaling="yarn", factor=4.0, original=512)
    w = [1 + 0.2 * torch.randn(dim, device="cuda", generator=gen) for _ in "qk"]
    plain, scale = Plain(rope, *w), dim ** -0.5

    def project(tokens):
        return torch.randn((tokens, hq + 2 * hkv, dim), device="cuda", generator=gen).to(dtype).split([hq, hkv, hkv], 1)

    def new_tokens(seq, counts):
        """extend, rotate and write; the queries."""
        kv.extend(i32(seq), i32(counts))
        q, k, v = project(sum(counts))
        offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), device="cuda")
        for s, a, b in zip(seq, offsets.tolist(), offsets.tolist()[1:]):
            plain.add(s, q[a:b], k[a:b], v[a:b])
        return kv.write_rotated(0, i32(seq), offsets, q, k, v, rope, *w), offsets

    def near(out, s, last):
        want, spread, reach = plain.attend(s, last, scale)
        # The bounds of the attention itself, and: queries and keys are rounded to their type after rotation (each logit is off by
        # at most twice a rounding of its reach), values of 8 bits by 2^-4 of themselves.
        off = km.bounds(spread, reach, dim, kind, "f16" if kind == "f16" else "bf16")[0]
        one = km.UNIT["f16" if kind == "f16" else "bf16"]
        keys = 2.0 ** -4 if kind == "e4m3" else one
        off = off + ((2 * (one + keys) * reach)[..., None] + (2.0 ** -4 if kind == "e4m3" else 0)) * spread + (0.03 * 2.0 ** -10 if kind == "e4m3" else 0)
        d = (out.double() - want).abs()
        assert bool((d <= off).all()), float((d / off).max())

    prefix, rests = 333, [1, 40, 7, 130, 16]
    q, offsets = new_tokens([0], [prefix])
    out, _ = kv.attend_prompt(0, q, offsets, scale, seq=i32([0]))
    kv.sync()
    near(out, 0, prefix)
    seq = [1, 2, 3, 4, 5]
    kv.fork(i32([0] * 5), i32(seq), i32([prefix] * 5))
    for s in seq:
        plain.fork(0, s, prefix)
    q, offsets = new_tokens(seq, rests)
    out, lse = kv.attend_prompt(0, q, offsets, scale, seq=i32(seq))
    kv.sync()
    for s, a, b in zip(seq, offsets.tolist(), offsets.tolist()[1:]):
        near(out[a:b], s, b - a)
    for _ in range(3):
        q, _ = new_tokens(seq, [1] * 5)
        out, lse = kv.attend_shared(0, q, i32([0, 5]), scale, seq=i32(seq), least=0)
        alone, lse1 = kv.attend(0, q, scale, seq=i32(seq))
        kv.sync()
        for i, s in enumerate(seq):
            near(out[i:i + 1], s, 1)
        assert torch.allclose(out.float(), alone.float(), atol=2.0 ** -7, rtol=2.0 ** -7) and torch.allclose(lse, lse1, atol=1e-4)


def test_two_caches_at_once():
    """Calls of two handles on two streams, overlapping: each has scratch of its own."""
    from test_gpu_kv_attend import make, query
    caches = [make([3000, 500, 40, 1200], 2, dim, 16, kind, seed=i) for i, (dim, kind) in enumerate([(128, "bf16"), (64, "f16")])]
    counts, o = [700, 500, 3, 64], torch.tensor([0, 700, 1200, 1203, 1267], device="cuda")
    queries = [query(1267, 14, c.dim, c.k.dtype) for c in caches]
    want = []
    for c, q in zip(caches, queries):
        want.append((c.attend_prompt(0, q, o), c.attend_shared(0, q[:4].contiguous(), i32([0, 4]), least=0)))
        c.sync()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in caches]
    for c, s in zip(caches, streams):
        c.set_stream(s)
    got = [[], []]
    for _ in range(20):
        for i, (c, q) in enumerate(zip(caches, queries)):
            with torch.cuda.stream(streams[i]):
                got[i].append((c.attend_prompt(0, q, o), c.attend_shared(0, q[:4], i32([0, 4]), least=0)))
    torch.cuda.synchronize()
    for c, results, w in zip(caches, got, want):
        c.sync()
        for r in results:
            for a, b in zip(r, w):
                assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_many_short_sequences_and_many_groups():
    """More items than a CTA's threads, one to three tokens each; groups of two."""
    from test_gpu_kv_attend import check, make, query
    rng = np.random.default_rng(0)
    n = 3001
    lengths = rng.integers(1, 40, n).tolist()
    counts = [min(x, int(y)) for x, y in zip(lengths, rng.integers(0, 4, n))]
    c = make(lengths, 1, 64, 8, "bf16")
    q = query(sum(counts), 4, 64, torch.bfloat16)
    o = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), device="cuda")
    got = c.attend_prompt(0, q, o)
    c.sync()
    some = rng.choice(n, 200, replace=False)
    rows = torch.cat([torch.arange(int(o[s]), int(o[s + 1])) for s in some]).cuda()
    part = torch.tensor(np.concatenate([[0], np.cumsum([counts[s] for s in some])]), device="cuda")
    rm.check(c, 0, q[rows], part, 0.125, (got[0][rows], got[1][rows]), i32(some))
    q = query(2 * n, 4, 64, torch.bfloat16)
    seq = i32(np.repeat(np.arange(n), 2))
    out, lse = c.attend_shared(0, q, i32(range(0, 2 * n + 1, 2)), seq=seq, least=0)
    alone, lse1 = c.attend(0, q, seq=seq)
    c.sync()
    assert torch.allclose(out.float(), alone.float(), atol=2.0 ** -7, rtol=2.0 ** -6) and torch.allclose(lse, lse1, atol=1e-4)
    check(c, 0, q[:64], 0.125, (out[:64], lse[:64]), seq[:64])
