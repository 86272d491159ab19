"""Operators of the paged key-value cache that handle many query rows together, and the way in of what it holds, as they are
measured: what a node does with a layer's queries, keys and values when requests hit its cached prefixes.

A case's ``kind`` is a pass:

  rotate   queries and keys of new tokens are normed for each head and rotated to their positions, which their sequences'
           lengths say; keys and values are written to the cache, the queries are returned
  prompt   the new tokens of every sequence attend over what it holds, each up to itself: cached tokens and their own
  shared   one new token of every row of a batch attends over its cached tokens; groups of rows begin with the same
           pages (a prefix that they were forked from), the rest of each row's tokens is its own

Keys and values are [layers, pages, tokens a page, kv heads, head dim]; with ``order`` "head" a page stores each head's
tokens together, with "token" each token's heads.  Lengths run from ``lo`` to ``hi``, evenly over their logarithm.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f16": 2, "e4m3": 1}
_EPS = 1e-6
_THETA = 10000.0
# Positions stretched for long contexts: what they were trained for, and how many times that they now reach.
_ORIGINAL, _FACTOR = 8192, 16.0


def listed():
    return [
        # A decode step of an ordinary batch, one layer: latency.
        dict(name="rotate, 33 x 1 token", kind="rotate", n=33, lo=256, hi=1152, new_lo=1, new_hi=1, hq=14, hkv=2, d=64, page=16,
             type="bf16", order="head", rot=64, pairs=False, scaling="none", norm=False),
        # Whole prompts, heads normed, positions scaled by parts of the spectrum, kept in 8 bits.
        dict(name="rotate, 61 prompts in 8 bits", kind="rotate", n=61, lo=1, hi=64, new_lo=128, new_hi=4224, hq=64, hkv=8, d=128,
             page=32, type="e4m3", order="head", rot=128, pairs=False, scaling="by_parts", norm=True),
        # A few long sequences go on, half of each head rotated in interleaved pairs, heads inside tokens.
        dict(name="rotate, far positions", kind="rotate", n=5, lo=1000, hi=120000, new_lo=1, new_hi=701, hq=24, hkv=24, d=80, page=1,
             type="f16", order="token", rot=40, pairs=True, scaling="yarn", norm=True),
        # A prompt of the mean length of the few-shot workload that hits nothing, alone on its node.
        dict(name="prompt, 1 x 540 tokens", kind="prompt", n=1, lo=1, hi=1, new_lo=540, new_hi=540, hq=14, hkv=2, d=64, page=16,
             type="bf16", order="head", window=0, empty=0),
        # An ordinary batch of requests with cached prefixes.
        dict(name="prompt, 16 on prefixes", kind="prompt", n=16, lo=2, hi=1024, new_lo=32, new_hi=1024, hq=32, hkv=8, d=128, page=16,
             type="bf16", order="head", window=0, empty=0),
        # A piece of a very long prompt, after the pieces before it.
        dict(name="prompt, 4,096 tokens after 12,288", kind="prompt", n=1, lo=12288, hi=12288, new_lo=4096, new_hi=4096, hq=40, hkv=8,
             d=128, page=64, type="f16", order="token", window=0, empty=0),
        # A few tokens each (drafts that are checked), under a sliding window, an odd head size, some rows with nothing new.
        dict(name="prompt, 1 to 9 tokens, window of 1,000", kind="prompt", n=191, lo=1, hi=8191, new_lo=1, new_hi=9, hq=24, hkv=24, d=80,
             page=1, type="bf16", order="token", window=1000, empty=7),
        # Large heads over a cache in 8 bits, pages that end inside any tile.
        dict(name="prompt, heads of 256 in 8 bits", kind="prompt", n=7, lo=1, hi=700, new_lo=100, new_hi=900, hq=32, hkv=2, d=256,
             page=100, type="e4m3", order="head", window=0, empty=0),
        # A decode step of the few-shot workload's requests on one instruction prefix.
        dict(name="shared, 64 on one prefix", kind="shared", n=64, groups=1, alone=0, lo=1024, hi=1024, own_lo=32, own_hi=128, hq=14,
             hkv=2, d=64, page=16, type="bf16", order="head", window=0),
        # A large batch on prefixes of skewed popularity, in 8 bits.
        dict(name="shared, 256 on 8 prefixes in 8 bits", kind="shared", n=256, groups=8, alone=0, lo=512, hi=8192, own_lo=32, own_hi=1152,
             hq=64, hkv=8, d=128, page=32, type="e4m3", order="head", window=0),
        # One long document that many requests ask about, five query heads a kv head, heads inside tokens.
        dict(name="shared, 200 on one of 8,192 tokens", kind="shared", n=200, groups=1, alone=0, lo=8192, hi=8192, own_lo=1, own_hi=513,
             hq=40, hkv=8, d=128, page=16, type="f16", order="token", window=0),
        # Many small groups and rows that share nothing, under a window that leaves some groups nothing shared to see.
        dict(name="shared, 37 groups, window of 1,000", kind="shared", n=150, groups=37, alone=20, lo=100, hi=5000, own_lo=1, own_hi=1500,
             hq=12, hkv=4, d=96, page=8, type="bf16", order="head", window=1000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "prompt", "prompt", "shared", "shared"])
    c = dict(kind=kind, type=rng.choice(["bf16", "f16", "e4m3"]), order=rng.choice(["head", "token"]),
             page=rng.choice([1, 8, 16, 16, 32, 64, 100]), hkv=rng.choice([1, 2, 4, 8]))
    hkv, group = c["hkv"], rng.choice([1, 2, 4, 5, 7, 8, 8, 12, 16])
    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    c.update(hq=hkv * group, d=d)
    if kind == "rotate":
        new_hi = rng.choice([1, 1, _log(rng, 2, 4224)])
        rot = rng.choice([d, d, d, d // 2, d // 4])
        # (no more values than the largest listed case has)
        n = max(1, min(_log(rng, 1, 512), 700_000_000 // (d * (c["hq"] + 2 * hkv) * new_hi)))
        return dict(c, n=n, lo=1, hi=min(_log(rng, 2, 120000), 20_000_000 // n), new_lo=max(1, new_hi // 20), new_hi=new_hi, rot=rot,
                    pairs=rng.random() < 0.4, scaling=rng.choice(["none", "none", "linear", "ntk", "by_parts", "yarn"]),
                    norm=rng.random() < 0.6)
    window = rng.choice([0, 0, 0, 128, 1000, 4096])
    if kind == "prompt":
        new_hi = _log(rng, 1, 4096)
        hi = _log(rng, 1, 16384)
        # (padded logits, products and keys: no more than the largest listed cases pad to)
        cost = max(c["hq"] * new_hi, 4 * hkv * d) * (hi + new_hi)
        most = 40 * 4096 * 14336
        while cost * d > most * 128:
            hi, new_hi = max(1, hi // 2), max(1, new_hi // 2)
            cost = max(c["hq"] * new_hi, 4 * hkv * d) * (hi + new_hi)
        n = max(1, min(_log(rng, 1, 256), most * 128 // (cost * max(d, 128))))
        return dict(c, n=n, lo=max(1, int(hi * rng.choice([0.01, 0.25, 1.0]))), hi=hi, new_lo=max(1, int(new_hi * rng.choice([0.05, 0.3, 1.0]))),
                    new_hi=new_hi, window=window, empty=rng.choice([0, 0, n // 6]))
    hi, own_hi = _log(rng, 16, 32768), _log(rng, 1, 2048)
    n = max(2, min(_log(rng, 2, 512), 256 * 9344 * 8 * 128 // ((hi + own_hi + c["page"]) * hkv * max(d, 8 * group))))
    groups = max(1, min(_log(rng, 1, 40), n // 2))
    return dict(c, n=n, groups=groups, alone=rng.choice([0, 0, min(n - 2 * groups, n // 5)]), lo=max(1, int(hi * rng.choice([0.1, 0.5, 1.0]))), hi=hi,
                own_lo=max(1, own_hi // 20), own_hi=own_hi, window=window)


# ---- sizes that a case fixes ------------------------------------------------------------------------------

def _spread(n, lo, hi):
    """n lengths from lo to hi, evenly over their logarithm (a single one: hi)."""
    u = (np.arange(n) + 0.5) / n if n != 1 else np.ones(1)
    return np.clip(np.rint(lo * (hi / lo) ** u), lo, hi).astype(np.int64)


def _mixed(x):
    """The same values in an order of their own, the same every time."""
    return x[np.argsort((np.arange(len(x)) + 1) * 0.6180339887 % 1.0)]


def _pages(length, page):
    return -(-length // page)


def _sizes(c):
    """A case's lengths and counts; the seed says only which sequence has which."""
    s, n = {}, c["n"]
    if c["kind"] != "shared":
        s["before"], s["count"] = _spread(n, c["lo"], c["hi"]), _mixed(_spread(n, c["new_lo"], c["new_hi"]))
        if c["kind"] == "prompt":
            s["count"][:c["empty"]] = 0
            s["before"][:c["empty"] // 2] = 0
        s["length"] = s["before"] + s["count"]
        return s
    # Popularity falls with a prefix's number; every group has two rows at least.
    rows, k = n - c["alone"], c["groups"]
    share = 1 / (np.arange(k) + 1.0)
    size = 2 + np.floor((rows - 2 * k) * share / share.sum()).astype(np.int64)
    size[0] += rows - size.sum()
    prefix = _mixed(_spread(k, c["lo"], c["hi"]))
    s["size"] = np.concatenate([size, np.ones(c["alone"], np.int64)])
    s["shared"] = np.concatenate([prefix // c["page"] * c["page"], np.zeros(c["alone"], np.int64)])  # (whole pages)
    tail = np.concatenate([prefix % c["page"], _mixed(_spread(c["alone"], c["lo"], c["hi"]))])
    s["own"] = _mixed(_spread(n, c["own_lo"], c["own_hi"])) + np.repeat(tail, s["size"])
    s["length"] = np.repeat(s["shared"], s["size"]) + s["own"]
    return s


def work(c):
    s, b = _sizes(c), _BYTES[c["type"]]
    n, p, hq, hkv, d = c["n"], c["page"], c["hq"], c["hkv"], c["d"]
    if c["kind"] == "rotate":
        new = int(s["count"].sum())
        return {"bytes": new * d * (2 * 2 * hq + 2 * hkv * (2 + b)) + 16 * n + 4 * int(_pages(s["count"], p).sum()),
                "flops": new * (hq + hkv) * (4 * d * c["norm"] + 3 * c["rot"])}
    row = 2 * hkv * d * b
    if c["kind"] == "prompt":
        begin = np.maximum(s["before"] + 1 - c["window"], 0) if c["window"] else np.zeros(n, np.int64)
        held = np.where(s["count"] > 0, s["length"] - begin, 0)
        whole = s["before"] * s["count"] + s["count"] * (s["count"] + 1) // 2   # (query, key) pairs
        if c["window"]:
            # Token j of a sequence sees min(before + j + 1, window).
            free = np.clip(c["window"] - s["before"], 0, s["count"])            # tokens that the window does not cut
            whole = free * s["before"] + free * (free + 1) // 2 + (s["count"] - free) * c["window"]
        new = int(s["count"].sum())
        return {"bytes": int(held.sum()) * row + 4 * int(_pages(held, p).sum()) + new * (4 * hq * d + 4 * hq) + 16 * n,
                "flops": 4 * int(whole.sum()) * hq * d}
    begin = np.maximum(s["length"] - c["window"], 0) if c["window"] else np.zeros(n, np.int64)
    shared = np.repeat(s["shared"], s["size"])
    first = np.minimum.reduceat(begin, np.concatenate([[0], np.cumsum(s["size"])[:-1]]))
    tokens = int(np.maximum(s["shared"] - first, 0).sum() + (s["length"] - np.maximum(begin, shared)).sum())
    seen = int((s["length"] - begin).sum())
    return {"bytes": tokens * row + 4 * int(_pages(s["length"] - begin, p).sum()) + n * (4 * hq * d + 4 * hq + 8),
            "flops": 4 * seen * hq * d}


def _inv_freq(rot, scaling):
    """(radians a position of each pair, what cos and sin are multiplied by), in 64 bits."""
    j = np.arange(rot // 2, dtype=np.float64)
    theta = _THETA * _FACTOR ** (rot / (rot - 2)) if scaling == "ntk" else _THETA
    f = theta ** (-2 * j / rot)
    if scaling == "linear":
        return f / _FACTOR, 1.0
    if scaling == "by_parts":   # pairs that turn less than once in the original length are stretched, above 4 turns kept
        keep = np.clip((_ORIGINAL * f / (2 * math.pi) - 1.0) / (4.0 - 1.0), 0, 1)
        return f * keep + f / _FACTOR * (1 - keep), 1.0
    if scaling == "yarn":       # the same with a ramp over the pairs' numbers, from 32 turns to 1
        at = [rot * math.log(_ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(_THETA)) for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        keep = 1 - np.clip((j - lo) / max(hi - lo, 1e-3), 0, 1)
        return f * keep + f / _FACTOR * (1 - keep), 0.1 * math.log(_FACTOR) + 1
    return f, 1.0


# ---- inputs -------------------------------------------------------------------------------------------------

def _bytes(x):
    """A tensor of an 8-bit type by its bytes (indexing does not know the type itself)."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _pool(c, n_pages, g):
    """Keys or values of a pool, all pages with something in them."""
    shape = (1, n_pages, c["hkv"], c["page"], c["d"]) if c["order"] == "head" else (1, n_pages, c["page"], c["hkv"], c["d"])
    x = torch.empty(shape, dtype=torch.bfloat16 if c["type"] == "e4m3" else _TYPES[c["type"]], device="cuda").normal_(generator=g)
    if c["type"] == "e4m3":
        x = x.mul(30).to(torch.float8_e4m3fn)   # (what scales of about 1/30 make of it)
    return x.permute(0, 1, 3, 2, 4) if c["order"] == "head" else x


def prepare(case, seed):
    c, s = case, _sizes(case)
    r = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, p, n = c["kind"], c["page"], c["n"]
    if kind == "shared":
        order = r.permutation(n)                      # the batch's row i is sequence order[i]
        group = np.repeat(np.arange(len(s["size"])), s["size"])
        common = s["shared"][group] // p              # entries of row i that its group shares
        length = np.empty(n, np.int64)
        length[order] = s["length"]
        distinct = int((s["shared"] // p).sum() + (_pages(s["length"], p) - common).sum())
    else:
        order = r.permutation(n)                      # sequence i has the lengths of order[i]
        length = s["length"][order]
        distinct = int(_pages(length, p).sum())
    n_pages = distinct + max(8, distinct // 8)
    ids = r.permutation(n_pages)[:distinct].astype(np.int32)   # a sequence's pages lie anywhere in the pool
    used = _pages(length, p)
    table = np.zeros((n, max(int(used.max()), 1)), np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0

    def take(k):
        nonlocal at
        at += int(k)
        return ids[at - int(k):at]

    if kind == "shared":
        prefix = [take(x // p) for x in s["shared"]]
        for i in range(n):
            q, m = order[i], int(common[i])
            table[q, :m] = prefix[group[i]]
            table[q, m:used[q]] = take(used[q] - m)
    else:
        for q in range(n):
            table[q, :used[q]] = take(used[q])
    for q in range(n):
        np.add.at(refs, table[q, :used[q]], 1)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a).astype(t)).cuda()  # noqa: E731
    half = torch.float16 if c["type"] == "f16" else torch.bfloat16
    st = dict(kind=kind, page=p, k=_pool(c, n_pages, g), v=_pool(c, n_pages, g), table=dev(table, np.int32), length=dev(length, np.int32),
              refs=dev(refs, np.int32), k_scale=None, v_scale=None, window=c.get("window", 0), scale=c["d"] ** -0.5)
    if c["type"] == "e4m3":
        st["k_scale"], st["v_scale"] = (torch.rand((1, c["hkv"]), device="cuda", generator=g) * 0.03 + 0.02 for _ in "kv")
    if kind != "rotate":
        # What no sequence holds may be anything, NaN among it: free pages and the ends of last pages.
        free = dev(np.setdiff1d(np.arange(n_pages), ids), np.int64)
        part = np.nonzero(length % p)[0]
        last = dev(table[part, used[part] - 1], np.int64)
        tail = torch.arange(p, device="cuda")[None] >= dev(length[part] % p, np.int64)[:, None]
        junk = 0x7F if c["type"] == "e4m3" else math.nan
        for x in (_bytes(st["k"]), _bytes(st["v"])):
            x[0, free] = junk
            x[0, last] = torch.where(tail[:, :, None, None], junk, x[0, last]).to(x.dtype)
    if kind == "shared":
        st.update(seq=dev(order, np.int32), groups=dev(np.concatenate([[0], np.cumsum(s["size"])]), np.int32),
                  q=(3 * torch.randn((n, c["hq"], c["d"]), device="cuda", generator=g)).to(half))
    else:
        mix = r.permutation(n)                        # the order of the call's list
        count = s["count"][order][mix]
        tokens = int(count.sum())
        st.update(seq=dev(mix, np.int32), offsets=dev(np.concatenate([[0], np.cumsum(count)]), np.int64))
        if kind == "prompt":
            st["q"] = (3 * torch.randn((tokens, c["hq"], c["d"]), device="cuda", generator=g)).to(half)
        else:
            # One projection gives all heads of a token: queries, keys, values.
            x = torch.empty((tokens, c["hq"] + 2 * c["hkv"], c["d"]), dtype=half, device="cuda").normal_(generator=g)
            st["q"], st["new_k"], st["new_v"] = x.split([c["hq"], c["hkv"], c["hkv"]], 1)
            inv_freq, amplitude = _inv_freq(c["rot"], c["scaling"])
            st.update(inv_freq=torch.from_numpy(inv_freq).cuda(), amplitude=amplitude, pairs=c["pairs"], q_weight=None, k_weight=None)
            if c["norm"]:
                st["q_weight"], st["k_weight"] = (1 + 0.2 * torch.randn(c["d"], device="cuda", generator=g) for _ in "qk")
    if own:
        import paper_2606_17059_gb300 as gb
        st["cache"] = gb.KvCache(st["k"], st["v"], st["table"], st["length"], st["refs"], k_scale=st["k_scale"], v_scale=st["v_scale"])
        if kind == "rotate":
            how = {"none": {}, "linear": dict(factor=_FACTOR), "ntk": dict(factor=_FACTOR),
                   "by_parts": dict(factor=_FACTOR, original=_ORIGINAL, low=1.0, high=4.0),
                   "yarn": dict(factor=_FACTOR, original=_ORIGINAL, low=1.0, high=32.0)}[c["scaling"]]
            st["rope"] = gb.Rope(c["rot"], theta=_THETA, interleaved=c["pairs"], scaling=None if c["scaling"] == "none" else c["scaling"], **how)
    return st


# ---- the passes ---------------------------------------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    kv = st["cache"]
    if st["kind"] == "rotate":
        q = kv.write_rotated(0, st["seq"], st["offsets"], st["q"], st["new_k"], st["new_v"], st["rope"], st["q_weight"], st["k_weight"], _EPS)
        return dict(q=q, k=st["k"], v=st["v"])
    if st["kind"] == "prompt":
        out, lse = kv.attend_prompt(0, st["q"], st["offsets"], st["scale"], seq=st["seq"], window=st["window"])
    else:
        out, lse = kv.attend_shared(0, st["q"], st["groups"], st["scale"], seq=st["seq"], window=st["window"])
    return dict(out=out, lse=lse)


def _run_plain(st):
    return {"rotate": _plain_rotate, "prompt": _plain_prompt, "shared": _plain_shared}[st["kind"]](st)


def _each(counts):
    """For items that hold `counts` entries: the item of every entry, and its place among the item's."""
    which = torch.repeat_interleave(torch.arange(len(counts), device=counts.device), counts)
    return which, torch.arange(len(which), device=counts.device) - (counts.cumsum(0) - counts)[which]


def _plain_rotate(st):
    seq, count, page = st["seq"].long(), st["offsets"].diff(), st["page"]
    which, j = _each(count)
    pos = (st["length"][seq].long() - count)[which] + j
    angle = pos[:, None].double() * st["inv_freq"]
    cos, sin = ((st["amplitude"] * f(angle)).float()[:, None] for f in (torch.cos, torch.sin))
    rot = 2 * len(st["inv_freq"])

    def turned(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS) * weight
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if st["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1 if st["pairs"] else -2).flatten(-2)
        return torch.cat([y, x[..., rot:]], -1)

    at = st["table"][seq[which], pos // page].long()
    for x, new, scale in ((st["k"], turned(st["new_k"], st["k_weight"]), st["k_scale"]), (st["v"], st["new_v"], st["v_scale"])):
        if scale is not None:
            new = (new.float() / scale[0][:, None]).clamp(-448, 448)
        _bytes(x)[0, at, pos % page] = _bytes(new.to(x.dtype))
    return dict(q=turned(st["q"], st["q_weight"]).to(st["q"].dtype), k=st["k"], v=st["v"])


def _rows(st, x, scale, seq, seen):
    """Keys or values of the sequences, [n, kv heads, tokens, head dim] in 32 bits, zero where nothing of them is seen."""
    pos = torch.arange(seen.shape[1], device=seen.device)
    y = _bytes(x[0])[st["table"][seq][:, pos // st["page"]].long(), pos % st["page"]].view(x.dtype).float()
    y = torch.where(seen[:, :, None, None], y, 0.0)
    return (y if scale is None else y * scale[0][:, None]).permute(0, 2, 1, 3)


def _softmax_rows(x, values):
    """(result, lse) of logits whose masked places are -inf; rows of nothing else give 0 and -inf."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(top), 0.0, top))
    z = e.sum(-1, keepdim=True)
    out = torch.where(z > 0, torch.matmul(e, values) / torch.where(z > 0, z, 1.0), 0.0)
    return out, (top + torch.log(torch.where(z > 0, z, 1.0)))[..., 0]


def _plain_prompt(st):
    q, seq, count = st["q"], st["seq"].long(), st["offsets"].diff()
    length = st["length"][seq].long()
    n, (tokens, hq, d), hkv = len(seq), q.shape, st["k"].shape[3]
    which, j = _each(count)
    most = int(count.max())
    padded = torch.zeros((n, most, hq, d), device=q.device)
    padded[which, j] = q.float()
    padded = padded.view(n, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    pos = torch.arange(int(length.max()), device=q.device)
    mine = (length - count)[:, None] + torch.arange(most, device=q.device)       # [n, most]: a token's place
    seen = pos <= mine[:, :, None]
    if st["window"]:
        seen &= pos > mine[:, :, None] - st["window"]
    held = (pos < length[:, None]) & (count > 0)[:, None]
    x = torch.matmul(padded, _rows(st, st["k"], st["k_scale"], seq, held).transpose(2, 3)).view(n, hkv, hq // hkv, most, -1) * st["scale"]
    x = torch.where(seen[:, None, None], x, -math.inf).view(n, hkv, -1, len(pos))
    out, lse = _softmax_rows(x, _rows(st, st["v"], st["v_scale"], seq, held))
    out = out.view(n, hq, most, d).transpose(1, 2)[which, j]
    return dict(out=out.to(q.dtype), lse=lse.view(n, hq, most).transpose(1, 2)[which, j])


def _plain_shared(st):
    q, seq = st["q"], st["seq"].long()
    length = st["length"][seq].long()
    (n, hq, d), hkv = q.shape, st["k"].shape[3]
    pos = torch.arange(int(length.max()), device=q.device)
    seen = pos < length[:, None]
    if st["window"]:
        seen &= pos >= length[:, None] - st["window"]
    x = torch.matmul(q.float().view(n, hkv, hq // hkv, d), _rows(st, st["k"], st["k_scale"], seq, seen).transpose(2, 3)) * st["scale"]
    out, lse = _softmax_rows(torch.where(seen[:, None, None], x, -math.inf), _rows(st, st["v"], st["v_scale"], seq, seen))
    return dict(out=out.to(q.dtype).view(n, hq, d), lse=lse.view(n, hq))


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------

def _round_e4m3(y):
    """The nearest value with 3 bits after the leading one, exponents from -6, at most 448; ties to even."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def exact(case, seed):
    s = _sizes(case)
    size = case["hq"] * case["d"]
    if case["kind"] == "rotate" and int(s["count"].sum()) * size > 1 << 31:
        return None
    if case["kind"] == "prompt" and int((s["count"] * s["length"]).sum()) * size > 1 << 42:
        return None
    if case["kind"] == "shared" and int(s["length"].sum()) * size > 1 << 36:
        return None
    st = prepare(case, seed)
    return _exact_rotate(st) if case["kind"] == "rotate" else _exact_attend(st)


def _exact_rotate(st):
    seq, offsets, length, table = (st[x].tolist() for x in ("seq", "offsets", "length", "table"))
    pos, pages = [], []
    for i, s in enumerate(seq):
        first = length[s] - (offsets[i + 1] - offsets[i])
        pos += range(first, length[s])
        pages += [table[s][t // st["page"]] for t in range(first, length[s])]
    pos, pages = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in (pos, pages))
    half = len(st["inv_freq"])
    angle = torch.outer(pos.double(), st["inv_freq"])
    turn = torch.polar(torch.full_like(angle, st["amplitude"]), angle)[:, None]

    def turned(x, weight):
        x = x.double()
        if weight is not None:
            x = weight.double() * x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + _EPS).sqrt()
        if st["pairs"]:
            x[..., :2 * half] = torch.view_as_real(torch.view_as_complex(x[..., :2 * half].unflatten(-1, (half, 2)).contiguous()) * turn).flatten(-2)
        else:
            z = torch.complex(x[..., :half], x[..., half:2 * half]) * turn
            x[..., :half], x[..., half:2 * half] = z.real, z.imag
        return x

    done = {}
    for name, new, scale in (("k", turned(st["new_k"], st["k_weight"]), st["k_scale"]), ("v", st["new_v"].double(), st["v_scale"])):
        done[name] = st[name].double()
        if scale is not None:
            new = _round_e4m3(new / scale.double()[0][:, None])
        done[name][0, pages, pos % st["page"]] = new
    return dict(q=turned(st["q"], st["q_weight"]), **done)


def _exact_attend(st):
    q, page, window = st["q"].double(), st["page"], st["window"]
    tokens, hq, d = q.shape
    hkv = st["k"].shape[3]
    group = hq // hkv
    out, lse = torch.zeros_like(q), torch.full((tokens, hq), -math.inf, dtype=torch.float64, device=q.device)
    seq, length, table = st["seq"].tolist(), st["length"].tolist(), st["table"].tolist()
    offsets = st["offsets"].tolist() if "offsets" in st else list(range(len(seq) + 1))
    for i, s in enumerate(seq):
        a, b, end = offsets[i], offsets[i + 1], length[s]
        if a == b or end == 0:
            continue
        place = torch.arange(end - (b - a), end, device=q.device)          # of the new tokens
        begin = max(0, end - (b - a) + 1 - window) if window else 0
        at = torch.arange(begin, end, device=q.device)
        ids = torch.tensor(table[s][begin // page:-(-end // page)], device=q.device)
        cut = slice(begin % page, begin % page + end - begin)
        k, v = (_bytes(x)[0].index_select(0, ids).view(x.dtype).double().flatten(0, 1)[cut] for x in (st["k"], st["v"]))
        if st["k_scale"] is not None:
            k, v = k * st["k_scale"][0].double()[:, None], v * st["v_scale"][0].double()[:, None]
        hidden = at[None] > place[:, None]
        if window:
            hidden |= at[None] <= place[:, None] - window
        for h in range(hq):
            x = (st["scale"] * (q[a:b, h] @ k[:, h // group].T)).masked_fill_(hidden, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, 1)
            out[a:b, h] = torch.exp(x - lse[a:b, h, None]) @ v[:, h // group]
    return dict(out=out, lse=lse)
