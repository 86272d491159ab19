"""The paged key-value cache from its definition: lists and 64-bit arithmetic on the host, one sequence at a time."""
import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
# Half the distance of neighbouring values, relative to the value: b bits of significand (8, 11) are 2^(1 - b) apart.
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def ceil_div(a, b):
    return -(-a // b)


def e4m3(y):
    """Nearest value with a 4-bit significand, exponents from -6 (below: multiples of 2^-9), at most 448; ties to even."""
    y = np.asarray(y, np.float64)
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.clip(np.rint(y / step) * step, -448, 448)


class Model:
    """The state of a cache on the host.  k and v: float64 [layers, pages, page, heads, dim]."""

    def __init__(self, k, v, table, length, refs, k_scale=None, v_scale=None):
        self.k, self.v = (x.double().cpu().numpy().copy() for x in (k, v))
        self.table, self.length, self.refs = (x.cpu().numpy().copy() for x in (table, length, refs))
        self.page = k.shape[2]
        self.scale = [None if s is None else s.double().cpu().numpy() for s in (k_scale, v_scale)]

    def pages(self, s):
        return [int(p) for p in self.table[s, :ceil_div(int(self.length[s]), self.page)]]

    def extend(self, seq, count):
        was = self.refs.copy()
        free = [int(p) for p in np.nonzero(was == 0)[0]]
        for s, c in zip(seq, count):
            n = int(self.length[s])
            have, want, used = ceil_div(n, self.page), ceil_div(n + c, self.page), n % self.page
            if c and used and was[self.table[s, have - 1]] > 1:
                old, new = int(self.table[s, have - 1]), free.pop(0)
                self.k[:, new, :used], self.v[:, new, :used] = self.k[:, old, :used], self.v[:, old, :used]
                self.refs[old] -= 1
                self.refs[new] = 1
                self.table[s, have - 1] = new
            for e in range(have, want):
                self.table[s, e] = free.pop(0)
                self.refs[self.table[s, e]] = 1
            self.length[s] = n + c

    def write(self, layer, seq, offsets, k, v):
        for x, new, scale in ((self.k, k, self.scale[0]), (self.v, v, self.scale[1])):
            new = new.double().cpu().numpy()
            for i, s in enumerate(seq):
                m = int(offsets[i + 1] - offsets[i])
                for j in range(m):
                    t = int(self.length[s]) - m + j
                    row = new[:, int(offsets[i]) + j]
                    if scale is not None:
                        row = e4m3(row / scale[layer:layer + len(new), :, None])
                    x[layer:layer + len(new), self.table[s, t // self.page], t % self.page] = row

    def fork(self, src, dst, tokens):
        for a, b, n in zip(src, dst, tokens):
            for e in range(ceil_div(int(n), self.page)):
                self.table[b, e] = self.table[a, e]
                self.refs[self.table[a, e]] += 1
        for b, n in zip(dst, tokens):
            self.length[b] = n

    def trim(self, seq, to):
        for s, n in zip(seq, to):
            for p in self.pages(s)[ceil_div(int(n), self.page):]:
                self.refs[p] -= 1
            self.length[s] = n

    def compact(self):
        live = int((self.refs > 0).sum())
        holes = [p for p in range(live) if self.refs[p] == 0]
        movers = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        for a, b in zip(movers, holes):
            self.k[:, b], self.v[:, b] = self.k[:, a], self.v[:, a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        to = dict(zip(movers, holes))
        for s in range(len(self.length)):
            for e, p in enumerate(self.pages(s)):
                self.table[s, e] = to.get(p, p)

    def same(self, cache):
        """Compares a KvCache with the model: contents as they are, table entries within the lengths, lengths, refs."""
        for x, y in ((cache.k, self.k), (cache.v, self.v)):
            assert np.array_equal(x.double().cpu().numpy(), y, equal_nan=True)
        assert np.array_equal(cache.length.cpu().numpy(), self.length)
        assert np.array_equal(cache.refs.cpu().numpy(), self.refs)
        table = cache.table.cpu().numpy()
        for s in range(len(self.length)):
            assert [int(p) for p in table[s, :len(self.pages(s))]] == self.pages(s), s


def pool(layers, pages, page, heads, dim, kind, order, seed):
    """Random keys and values [layers, pages, page, heads, dim] stored in `order`: the dimensions from the outermost in."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = dict(l=layers, n=pages, t=page, h=heads)
    out = []
    for _ in "kv":
        x = torch.randn([size[o] for o in order] + [dim], device="cuda", generator=g)
        x = (x * 30).to(TYPES[kind]) if kind == "e4m3" else x.to(TYPES[kind])
        out.append(x.permute([order.index(o) for o in "lnth"] + [4]))
    return out


def attend(cache, layer, q, scale, seq=None, window=0):
    """(out, lse, spread, reach) in 64 bits, on the cache's device: spread = sum p |v|, reach = max |scale| sum |q| |k| over
    the tokens seen (both say how far roundings of their terms can carry)."""
    q = q.double()
    n, hq, dim = q.shape
    table, length = cache.table.tolist(), cache.length.tolist()
    page, heads = cache.k.shape[2], cache.heads
    out, spread = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((n, hq), -torch.inf, dtype=torch.float64, device=q.device)
    reach = torch.zeros((n, hq), dtype=torch.float64, device=q.device)
    for i, s in enumerate(range(n) if seq is None else seq.tolist()):
        rows = list(range(max(0, length[s] - window) if window else 0, length[s]))
        if not rows:
            continue
        at = torch.tensor([[table[s][t // page] for t in rows], [t % page for t in rows]], device=q.device)
        k, v = (x[layer].contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16)[at[0], at[1]].view(x.dtype).double()
                for x in (cache.k, cache.v))
        if cache.k_scale is not None:
            k, v = k * cache.k_scale[layer].double()[:, None], v * cache.v_scale[layer].double()[:, None]
        for h in range(heads):
            mine = slice(h * hq // heads, (h + 1) * hq // heads)
            x = scale * (q[i, mine] @ k[:, h].T)
            lse[i, mine] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            out[i, mine], spread[i, mine] = p @ v[:, h], p @ v[:, h].abs()
            reach[i, mine] = abs(scale) * (q[i, mine].abs() @ k[:, h].abs().T).amax(1)
    return out, lse, spread, reach


def bounds(spread, reach, dim, kind, out_kind):
    """How far out and lse may be off.  A logit is a sum of dim products held in 32 bits: at most dim * 2^-24 * reach off,
    and as much again for the products with scale and log2 e, doubled for the maximum that is taken off; exp of it is that
    much off, relatively, and 2^-21 for the function itself; a probability is rounded to the type of the product with v
    (f16 with 8-bit values), and the result to its own.  Sums of n terms in 32 bits in any order: covered by 2^-15 for the
    lengths here (their terms are positive, or bounded by spread)."""
    x = 4 * (dim + 4) * 2.0 ** -24 * reach + 2.0 ** -21
    if kind == "e4m3":
        x = x + 2 * dim ** 0.5 * 2.0 ** -12 * 2.0 ** -11 * reach  # (q in 11 bits relative to its row's largest value)
    p = UNIT["f16"] if kind == "e4m3" else UNIT[kind]
    return (x[..., None] * 2 + p + UNIT[out_kind] + 2.0 ** -15) * spread + 2.0 ** -24, x + 2.0 ** -15
