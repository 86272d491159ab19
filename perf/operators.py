"""The paged key-value cache's operators as they are measured: what a node that serves the requests routed to it does
with the pages behind its own trie.

A case's ``kind`` is a pass:

  attend   one new token of every sequence attends over its cached tokens
  append   new tokens join the sequences: pages are found, their keys and values of all layers written; the
           sequences then go back to the lengths they had, so that a pass can be repeated
  hit      requests whose prefix is cached: what the last pass forked is freed, each request forks the matched tokens of
           a cached sequence, takes room for the rest of its prompt (a shared, partly used page is copied) and writes it
  compact  half of the sequences leave, the others' pages move to the front of the pool, as many arrive again (the
           two halves take turns)

Keys and values are [layers, pages, tokens a page, kv heads, head dim]; with ``order`` "head" a page stores each head's
tokens together, with "token" each token's heads.  Lengths run from ``lo`` to ``hi``, evenly over their logarithm.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f16": 2, "e4m3": 1}


def listed():
    return [
        # A prompt of the mean length of the few-shot workload, alone on its node: launches and latency.
        dict(name="attend, 1 x 540 tokens", kind="attend", n=1, lo=540, hi=540, hq=14, hkv=2, d=64, page=16, type="bf16",
             order="head", window=0, empty=0),
        # A decode step of an ordinary batch (shared prefixes of 256 to 1,024 tokens and suffixes of 32 to 128).
        dict(name="attend, 64 ragged", kind="attend", n=64, lo=288, hi=1152, hq=14, hkv=2, d=64, page=16, type="bf16",
             order="head", window=0, empty=0),
        # One very long context: only its length gives the GPU work.
        dict(name="attend, 1 x 131,071 tokens", kind="attend", n=1, lo=131071, hi=131071, hq=32, hkv=8, d=128, page=64,
             type="bf16", order="head", window=0, empty=0),
        # Long-context prompts (4,096 to 32,768 tokens and a suffix), five query heads a kv head, heads inside tokens.
        dict(name="attend, 32 long", kind="attend", n=32, lo=4352, hi=33792, hq=40, hkv=8, d=128, page=16, type="f16",
             order="token", window=0, empty=0),
        # A large batch over a cache held in 8 bits (prefixes of 128 to 4,096 tokens).
        dict(name="attend, 256 in 8 bits", kind="attend", n=256, lo=128, hi=4224, hq=64, hkv=8, d=128, page=32, type="e4m3",
             order="head", window=0, empty=0),
        # A sliding window over token-wise pages, one kv head a query head, an odd head size, and rows not yet filled.
        dict(name="attend, window of 1,000", kind="attend", n=191, lo=1, hi=8191, hq=24, hkv=24, d=80, page=1, type="bf16",
             order="token", window=1000, empty=7),
        # A decode step's new tokens of all layers.
        dict(name="append, 33 x 1 token", kind="append", n=33, lo=256, hi=1152, new_lo=1, new_hi=1, layers=24, hkv=2, d=64,
             page=16, type="bf16", order="head"),
        # Whole prompts come in and are kept in 8 bits.
        dict(name="append, 61 prompts in 8 bits", kind="append", n=61, lo=1, hi=64, new_lo=128, new_hi=4224, layers=8, hkv=8,
             d=128, page=32, type="e4m3", order="head"),
        # A few requests that hit one of 57 shared prefixes.
        dict(name="hit, 24 requests", kind="hit", n=24, prefixes=57, lo=256, hi=1024, new_lo=32, new_hi=128, layers=24, hkv=2,
             d=64, page=16, type="bf16", order="head"),
        # Many requests on 512 prefixes whose popularity is skewed; large pages, so that shared ones are copied in part.
        dict(name="hit, 601 requests", kind="hit", n=601, prefixes=512, lo=128, hi=2048, new_lo=1, new_hi=128, layers=24, hkv=2,
             d=64, page=64, type="f16", order="token"),
        # A small node tidies up.
        dict(name="compact, 40 sequences", kind="compact", n=40, lo=256, hi=1152, layers=24, hkv=2, d=64, page=16, type="bf16",
             order="head"),
        # A large pool before a part of it is given back.
        dict(name="compact, 600 sequences", kind="compact", n=600, lo=256, hi=2176, layers=24, hkv=2, d=64, page=16,
             type="bf16", order="head"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "hit", "compact"])
    type_ = rng.choice(["bf16", "f16", "e4m3"])
    c = dict(kind=kind, type=type_, order=rng.choice(["head", "token"]), page=rng.choice([1, 8, 16, 16, 32, 64, 100]))
    if kind == "attend":
        hkv = rng.choice([1, 2, 4, 8])
        d = rng.choice([64, 64, 80, 96, 128, 128, 192, 256])
        group = rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16])
        # (the padded lengths of all sequences: no more keys than the largest listed case pads to)
        most = 32 * 33792 * 8 * 128 // (hkv * max(d, 8 * group))
        hi = min(_log(rng, 1, 131072), most)
        n = max(1, min(_log(rng, 1, 512), most // hi))
        return dict(c, n=n, lo=max(1, int(hi * rng.choice([0.03, 0.25, 1.0]))), hi=hi, hq=hkv * group, hkv=hkv, d=d,
                    window=rng.choice([0, 0, 0, 128, 1000, 4096]), empty=rng.choice([0, 0, n // 5]))
    hkv, d = rng.choice([(2, 64), (2, 64), (4, 96), (8, 128), (1, 256)])
    layers = rng.choice([1, 4, 12, 24])
    row = layers * hkv * d * _BYTES[type_]
    if kind == "append":
        new_hi = rng.choice([1, 1, _log(rng, 2, 4224)])
        n = max(1, min(_log(rng, 1, 512), (1 << 30) // (row * (new_hi + 600))))
        return dict(c, n=n, lo=1, hi=_log(rng, 2, 1152), new_lo=max(1, new_hi // 20), new_hi=new_hi, layers=layers, hkv=hkv, d=d)
    if kind == "hit":
        hi = _log(rng, 64, 2048)
        n = max(1, min(_log(rng, 1, 700), (3 << 28) // (row * (128 + 2 * c["page"]))))
        p = max(1, min(_log(rng, 1, 512), (3 << 28) // (row * hi)))
        return dict(c, n=n, prefixes=p, lo=max(1, hi // 10), hi=hi, new_lo=1, new_hi=_log(rng, 1, 128), layers=layers, hkv=hkv, d=d)
    hi = _log(rng, 64, 2176)
    n = max(2, min(_log(rng, 2, 600), (3 << 30) // (row * (hi + c["page"]))))
    return dict(c, n=n, lo=max(1, hi // 8), hi=hi, layers=layers, hkv=hkv, d=d)


# ---- sizes that a case fixes ------------------------------------------------------------------------------

def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly over their logarithm (a single one: hi)."""
    u = (np.arange(n) + 0.5) / n if n > 1 else np.ones(1)
    return np.clip(np.rint(lo * (hi / lo) ** u), lo, hi).astype(np.int64)


def _pages(length, page):
    return -(-length // page)


def _sizes(c):
    """A case's lengths and counts; the seed says only which sequence has which."""
    s = {}
    if c["kind"] == "attend":
        s["length"] = _spread(c["n"], c["lo"], c["hi"])
        s["length"][:c["empty"]] = 0
    elif c["kind"] == "append":
        s["length"], s["count"] = _spread(c["n"], c["lo"], c["hi"]), _spread(c["n"], c["new_lo"], c["new_hi"])[::-1].copy()
    elif c["kind"] == "hit":
        s["length"] = _spread(c["prefixes"], c["lo"], c["hi"])
        u = (np.arange(c["n"]) + 0.5) / c["n"]
        s["src"] = np.minimum((c["prefixes"] * u * u).astype(np.int64), c["prefixes"] - 1)  # few prefixes take most
        s["match"] = 1 + ((s["length"][s["src"]] - 1) * ((np.arange(c["n"]) + 1) * 0.6180339887 % 1.0)).astype(np.int64)
        s["count"] = _spread(c["n"], c["new_lo"], c["new_hi"])[::-1].copy()
    else:
        s["length"] = _spread(c["n"], c["lo"], c["hi"])
    return s


def work(c):
    s, b = _sizes(c), _BYTES[c["type"]]
    n, p = c["n"], c["page"]
    if c["kind"] == "attend":
        seen = np.minimum(s["length"], c["window"]) if c["window"] else s["length"]
        tokens = int(seen.sum())
        entries = int((_pages(s["length"], p) - (s["length"] - seen) // p).sum())
        return {"bytes": 2 * tokens * c["hkv"] * c["d"] * b + 4 * entries + n * (2 * c["hq"] * c["d"] * 2 + 4 * c["hq"] + 4),
                "flops": 4 * tokens * c["hq"] * c["d"]}
    row = 2 * c["layers"] * c["hkv"] * c["d"]  # values of a token
    if c["kind"] == "append":
        new = int(s["count"].sum())
        taken = int((_pages(s["length"] + s["count"], p) - _pages(s["length"], p)).sum())
        return {"bytes": new * row * (2 + b) + 16 * taken + 16 * n, "flops": 0}
    if c["kind"] == "hit":
        new, shared = int(s["count"].sum()), int(_pages(s["match"], p).sum())
        copied = int((s["match"] % p).sum())
        return {"bytes": new * row * (2 + b) + 2 * copied * row * b + 24 * shared + 24 * n, "flops": 0}
    pages = _pages(s["length"], p)
    moved = int(min(pages[0::2].sum(), pages[1::2].sum()))
    return {"bytes": 2 * moved * p * row * b + 16 * int(pages.sum()), "flops": 0}


# ---- inputs -------------------------------------------------------------------------------------------------

def _bytes(x):
    """A tensor of an 8-bit type by its bytes (indexing does not know the type itself)."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _pool(c, layers, n_pages, g):
    """Keys or values of a pool, all pages with something in them: an old occupant's, as in a pool in use."""
    shape = (layers, n_pages, c["hkv"], c["page"], c["d"]) if c["order"] == "head" else (layers, n_pages, c["page"], c["hkv"], c["d"])
    x = torch.empty(shape, dtype=torch.bfloat16 if c["type"] == "e4m3" else _TYPES[c["type"]], device="cuda").normal_(generator=g)
    if c["type"] == "e4m3":
        x = torch.cat([y.mul(30).to(torch.float8_e4m3fn) for y in x.split(1)])  # (what scales of about 1/30 make of it)
    return x.permute(0, 1, 3, 2, 4) if c["order"] == "head" else x


def prepare(case, seed):
    c, s = case, _sizes(case)
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    layers, kind = c.get("layers", 1), c["kind"]
    order = r.permutation(len(s["length"]))  # which row has which length
    length = s["length"][order]
    rows, used = len(length), _pages(length, c["page"])
    room = int(used.max(initial=0))  # pages of the longest row there will be
    spare = 0
    if kind == "append":
        count = s["count"][order]
        room = int(_pages(length + count, c["page"]).max())
        spare = int((_pages(length + count, c["page"]) - used).sum())
    elif kind == "hit":
        mix = r.permutation(c["n"])
        where = np.argsort(order)  # the row of a prefix
        src, match, count = where[s["src"][mix]], s["match"][mix], s["count"][mix]
        room = max(room, int(_pages(match + count, c["page"]).max()))
        spare = int((_pages(match + count, c["page"]) - _pages(match, c["page"]) + 1).sum())
        length = np.concatenate([length, np.zeros(c["n"], np.int64)])
        used = _pages(length, c["page"])
        rows += c["n"]
    total = int(used.sum())
    n_pages = total + spare + max(8, total // 8)
    # A pool that has been in use: a sequence's pages lie anywhere in it.
    ids = r.permutation(n_pages)[:total]
    if kind == "compact":
        ids = r.permutation(total + total // 8)[:total]
    table = np.zeros((rows, max(room, 1)), np.int32)
    at = np.concatenate([[0], np.cumsum(used)])
    for i in range(rows):
        table[i, :used[i]] = ids[at[i]:at[i + 1]]
    refs = np.zeros(n_pages, np.int32)
    refs[ids] = 1
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a).astype(t)).cuda()  # noqa: E731
    st = dict(kind=kind, page=c["page"], k=_pool(c, layers, n_pages, g), v=_pool(c, layers, n_pages, g), table=dev(table, np.int32),
              length=dev(length, np.int32), refs=dev(refs, np.int32), k_scale=None, v_scale=None)
    if c["type"] == "e4m3":
        st["k_scale"], st["v_scale"] = (torch.rand((layers, c["hkv"]), device="cuda", generator=g) * 0.03 + 0.02 for _ in "kv")
    half = torch.float16 if c["type"] == "f16" else torch.bfloat16
    if kind == "attend":
        # What the sequences do not hold may be anything, NaN among it: free pages and the ends of last pages.
        free = dev(np.setdiff1d(np.arange(n_pages), ids), np.int64)
        part = np.nonzero(length % c["page"])[0]
        last = dev(table[part, used[part] - 1], np.int64)
        tail = torch.arange(c["page"], device="cuda")[None] >= dev(length[part] % c["page"], np.int64)[:, None]
        junk = 0x7F if c["type"] == "e4m3" else math.nan
        for x in (_bytes(st["k"]), _bytes(st["v"])):
            x[0, free] = junk
            x[0, last] = torch.where(tail[:, :, None, None], junk, x[0, last]).to(x.dtype)
        st.update(q=(3 * torch.randn((rows, c["hq"], c["d"]), device="cuda", generator=g)).to(half), scale=c["d"] ** -0.5,
                  window=c["window"])
    elif kind == "append":
        seq = r.permutation(rows)
        st.update(seq=dev(seq, np.int32), count=dev(count[seq], np.int32), back=dev(length[seq], np.int32),
                  offsets=dev(np.concatenate([[0], np.cumsum(count[seq])]), np.int64))
    elif kind == "hit":
        dst = rows - c["n"] + r.permutation(c["n"])
        st.update(src=dev(src, np.int32), dst=dev(dst, np.int32), match=dev(match, np.int32), count=dev(count, np.int32),
                  none=torch.zeros(c["n"], dtype=torch.int32, device="cuda"),
                  offsets=dev(np.concatenate([[0], np.cumsum(count)]), np.int64))
    else:
        half_of = np.argsort(order)  # the row of each length, shortest first: the halves take every other one
        groups = [r.permutation(half_of[0::2]), r.permutation(half_of[1::2])]
        st.update(turn=0, groups=[dict(seq=dev(x, np.int32), none=torch.zeros(len(x), dtype=torch.int32, device="cuda"),
                                       count=dev(length[x], np.int32)) for x in groups])
    if kind in ("append", "hit"):
        tokens = int(st["offsets"][-1])
        st["new_k"], st["new_v"] = (torch.empty((layers, tokens, c["hkv"], c["d"]), dtype=half, device="cuda").normal_(generator=g)
                                    for _ in "kv")
    if own:
        import paper_2606_17059_gb300 as gb
        st["cache"] = gb.KvCache(st["k"], st["v"], st["table"], st["length"], st["refs"], k_scale=st["k_scale"],
                                 v_scale=st["v_scale"])
    return st


# ---- the passes ---------------------------------------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _state(st):
    return dict(k=st["k"], v=st["v"], table=st["table"], length=st["length"], refs=st["refs"])


def _run_own(st):
    kv = st["cache"]
    if st["kind"] == "attend":
        out, lse = kv.attend(0, st["q"], st["scale"], window=st["window"])
        return dict(out=out, lse=lse)
    if st["kind"] == "append":
        kv.extend(st["seq"], st["count"])
        kv.write(0, st["seq"], st["offsets"], st["new_k"], st["new_v"])
        kv.trim(st["seq"], st["back"])
    elif st["kind"] == "hit":
        kv.trim(st["dst"], st["none"])
        kv.fork(st["src"], st["dst"], st["match"])
        kv.extend(st["dst"], st["count"])
        kv.write(0, st["dst"], st["offsets"], st["new_k"], st["new_v"])
    else:
        gr = st["groups"][st["turn"]]
        st["turn"] ^= 1
        kv.trim(gr["seq"], gr["none"])
        kv.compact()
        kv.extend(gr["seq"], gr["count"])
    return _state(st)


def _run_plain(st):
    if st["kind"] == "attend":
        return _plain_attend(st)
    if st["kind"] == "append":
        _plain_extend(st, st["seq"], st["count"])
        _plain_write(st, st["seq"], st["offsets"], st["new_k"], st["new_v"])
        _plain_trim(st, st["seq"], st["back"])
    elif st["kind"] == "hit":
        _plain_trim(st, st["dst"], st["none"])
        _plain_fork(st, st["src"], st["dst"], st["match"])
        _plain_extend(st, st["dst"], st["count"])
        _plain_write(st, st["dst"], st["offsets"], st["new_k"], st["new_v"])
    else:
        gr = st["groups"][st["turn"]]
        st["turn"] ^= 1
        _plain_trim(st, gr["seq"], gr["none"])
        _plain_compact(st)
        _plain_extend(st, gr["seq"], gr["count"])
    return _state(st)


def _plain_attend(st):
    q, length, page = st["q"], st["length"].long(), st["page"]
    n, hq, d = q.shape
    hkv = st["k"].shape[3]
    pos = torch.arange(int(length.max()) if n else 0, device=q.device)
    first = (length - st["window"]).clamp(min=0) if st["window"] else torch.zeros_like(length)
    seen = (pos >= first[:, None]) & (pos < length[:, None])
    at = st["table"][:, pos // page].long()

    def rows(x, scale):
        y = _bytes(x[0])[at, pos % page].view(x.dtype).float()
        y = torch.where(seen[:, :, None, None], y, 0.0)
        return (y if scale is None else y * scale[0][:, None]).permute(0, 2, 1, 3)

    x = torch.matmul(q.float().view(n, hkv, hq // hkv, d), rows(st["k"], st["k_scale"]).transpose(2, 3)) * st["scale"]
    x = torch.where(seen[:, None, None], x, -math.inf)
    some = seen.any(1)[:, None, None, None]
    top = torch.where(some, x.amax(-1, keepdim=True) if len(pos) else 0.0, 0.0)
    e = torch.exp(x - top)
    z = e.sum(-1, keepdim=True)
    out = torch.where(some, torch.matmul(e, rows(st["v"], st["v_scale"])) / z, 0.0)
    return dict(out=out.to(q.dtype).view(n, hq, d), lse=(top + torch.log(z)).view(n, hq))


def _each(counts):
    """For items that hold `counts` entries: the item of every entry, and its place among the item's."""
    which = torch.repeat_interleave(torch.arange(len(counts), device=counts.device), counts)
    return which, torch.arange(len(which), device=counts.device) - (counts.cumsum(0) - counts)[which]


def _plain_extend(st, seq, count):
    page, table, refs, seq = st["page"], st["table"], st["refs"], seq.long()
    old = st["length"][seq].long()
    have, want = _pages(old, page), _pages(old + count, page)
    last = table[seq, (have - 1).clamp(min=0)].long()
    split = (old % page != 0) & (count > 0) & (refs[last] > 1)  # partly used and shared: it gets a copy of its own
    which, j = _each(want - have + split)
    taken = (refs == 0).nonzero()[:, 0][:len(which)]
    table[seq[which], (have - split.long())[which] + j] = taken.int()
    refs[taken] = 1
    src = last[split]
    refs.index_add_(0, src, torch.full_like(src, -1).int())
    dst = table[seq[split], have[split] - 1].long()
    kept = torch.arange(page, device=seq.device) < (old % page)[split][:, None]
    for x in (_bytes(st["k"]), _bytes(st["v"])):
        x[:, dst] = torch.where(kept[None, :, :, None, None], x[:, src], x[:, dst])
    st["length"][seq] = (old + count).int()


def _plain_write(st, seq, offsets, new_k, new_v):
    page, count = st["page"], offsets.diff()
    which, j = _each(count)
    pos = (st["length"][seq.long()] - count)[which] + j
    at = st["table"][seq.long()[which], pos // page].long()
    for x, new, scale in ((st["k"], new_k, st["k_scale"]), (st["v"], new_v, st["v_scale"])):
        if scale is not None:
            new = (new.float() / scale[:, None, :, None]).clamp(-448, 448).to(x.dtype)
        _bytes(x)[:, at, pos % page] = _bytes(new)


def _plain_trim(st, seq, to):
    page, seq = st["page"], seq.long()
    keep = _pages(to.long(), page)
    which, j = _each(_pages(st["length"][seq].long(), page) - keep)
    gone = st["table"][seq[which], keep[which] + j].long()
    st["refs"].index_add_(0, gone, torch.full_like(gone, -1).int())
    st["length"][seq] = to


def _plain_fork(st, src, dst, match):
    which, j = _each(_pages(match.long(), st["page"]))
    shared = st["table"][src.long()[which], j]
    st["table"][dst.long()[which], j] = shared
    st["refs"].index_add_(0, shared.long(), torch.ones_like(shared))
    st["length"][dst.long()] = match


def _plain_compact(st):
    refs, page = st["refs"], st["page"]
    live = refs > 0
    low = torch.arange(len(refs), device=refs.device) < live.sum()
    src, dst = (live & ~low).nonzero()[:, 0], (~live & low).nonzero()[:, 0]
    for x in (_bytes(st["k"]), _bytes(st["v"])):
        x[:, dst] = x[:, src]
    to = torch.arange(len(refs), device=refs.device, dtype=torch.int32)
    to[src] = dst.int()
    used = torch.arange(st["table"].shape[1], device=refs.device) < _pages(st["length"].long(), page)[:, None]
    st["table"].copy_(torch.where(used, to[st["table"].long()], st["table"]))
    refs[dst] = refs[src]
    refs[src] = 0


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------

def _round_e4m3(y):
    """The nearest value with 3 bits after the leading one, exponents from -6, at most 448; ties to even."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def exact(case, seed):
    values = sum(math.prod(x) for x in [(case.get("layers", 1), case["hkv"], case["d"])])
    s = _sizes(case)
    if case["kind"] != "attend" and int(s["length"].sum() + s.get("count", np.zeros(1)).sum()) * values > 1 << 28:
        return None
    if case["kind"] == "attend" and int(s["length"].sum()) * case["hq"] * case["d"] > 1 << 33:
        return None
    st = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(st)
    return _exact_pages(st)


def _exact_attend(st):
    q = st["q"].double()
    n, hq, d = q.shape
    hkv = st["k"].shape[3]
    out, lse = torch.zeros_like(q), torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    table, length = st["table"].tolist(), st["length"].tolist()
    for i in range(n):
        end = length[i]
        begin = max(0, end - st["window"]) if st["window"] else 0
        if begin == end:
            continue
        ids = torch.tensor(table[i][begin // st["page"]:-(-end // st["page"])], device=q.device)
        cut = slice(begin % st["page"], begin % st["page"] + end - begin)
        k, v = (_bytes(x)[0].index_select(0, ids).view(x.dtype).double().flatten(0, 1)[cut] for x in (st["k"], st["v"]))
        if st["k_scale"] is not None:
            k, v = k * st["k_scale"][0].double()[:, None], v * st["v_scale"][0].double()[:, None]
        for h in range(hkv):
            mine = slice(h * hq // hkv, (h + 1) * hq // hkv)
            x = st["scale"] * (q[i, mine] @ k[:, h].T)
            lse[i, mine] = torch.logsumexp(x, 1)
            out[i, mine] = torch.exp(x - lse[i, mine, None]) @ v[:, h]
    return dict(out=out, lse=lse)


def _exact_pages(st):
    page, refs, length = st["page"], st["refs"].tolist(), st["length"].tolist()
    table = st["table"].tolist()
    k, v = st["k"].double(), st["v"].double()

    def extend(seq, count):
        free = [p for p, x in enumerate(refs) if x == 0]
        free.reverse()
        was = list(refs)
        for s, c in zip(seq, count):
            if c and length[s] % page and was[table[s][length[s] // page]] > 1:
                old, new, t = table[s][length[s] // page], free.pop(), length[s] % page
                k[:, new, :t], v[:, new, :t] = k[:, old, :t], v[:, old, :t]
                table[s][length[s] // page] = new
                refs[old] -= 1
                refs[new] = 1
            for e in range(-(-length[s] // page), -(-(length[s] + c) // page)):
                table[s][e] = free.pop()
                refs[table[s][e]] = 1
            length[s] += c

    def write(seq, offsets):
        for new, scale, x in ((st["new_k"], st["k_scale"], k), (st["new_v"], st["v_scale"], v)):
            new = new.double()
            if scale is not None:
                new = _round_e4m3(new / scale.double()[:, None, :, None])
            ids, slots = [], []
            for i, s in enumerate(seq):
                begin = length[s] - (offsets[i + 1] - offsets[i])
                ids += [table[s][t // page] for t in range(begin, length[s])]
                slots += [t % page for t in range(begin, length[s])]
            x[:, torch.tensor(ids, device=x.device), torch.tensor(slots, device=x.device)] = new

    def trim(seq, to):
        for s, t in zip(seq, to):
            for e in range(-(-t // page), -(-length[s] // page)):
                refs[table[s][e]] -= 1
            length[s] = t

    if st["kind"] == "append":
        seq = st["seq"].tolist()
        extend(seq, st["count"].tolist())
        write(seq, st["offsets"].tolist())
        trim(seq, st["back"].tolist())
    elif st["kind"] == "hit":
        dst = st["dst"].tolist()
        for a, b, t in zip(st["src"].tolist(), dst, st["match"].tolist()):
            for e in range(-(-t // page)):
                table[b][e] = table[a][e]
                refs[table[a][e]] += 1
            length[b] = t
        extend(dst, st["count"].tolist())
        write(dst, st["offsets"].tolist())
    else:
        gr = st["groups"][st["turn"]]
        trim(gr["seq"].tolist(), gr["none"].tolist())
        n_live = sum(x > 0 for x in refs)
        holes = [p for p in range(n_live) if refs[p] == 0]
        to = dict(zip([p for p in range(n_live, len(refs)) if refs[p] > 0], holes))
        for a, b in to.items():
            k[:, b], v[:, b] = k[:, a], v[:, a]
            refs[b], refs[a] = refs[a], 0
        for s, row in enumerate(table):
            for e in range(-(-length[s] // page)):
                row[e] = to.get(row[e], row[e])
        extend(gr["seq"].tolist(), gr["count"].tolist())
    whole = lambda a, like: torch.tensor(a, dtype=like.dtype, device=like.device)  # noqa: E731
    return dict(k=k, v=v, table=whole(table, st["table"]), length=whole(length, st["length"]), refs=whole(refs, st["refs"]))
