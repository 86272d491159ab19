"""One node of the paper's cluster around its router: Algorithm 1 with the key-value cache behind the node's own trie.

Requests arrive in batches and are routed.  Those that stay on the node (tree 0, its own LRU trie) are served from the
paged cache: the matched tokens of a cached prompt are forked, the rest is appended, new tokens are decoded one by one with
attention over the cache, and the finished prompt stays cached.  When the pages run short, the least recently used
tokens leave the trie (EvictLRUTrie) and the same tokens leave the cache (EvictKVCache); the pages are moved together at the
end.  The language model is a stand-in without weights of its own: a token's queries, keys and values are fixed functions of
its id, its position and the layer, and the next token is read off the last layer's attention.  It gives the cache real work
whose results can be recomputed from the tokens alone (--check).

  python examples/serve_node.py [--batches 6] [--requests 48] [--decode 4] [--dtype bfloat16|float16|float8_e4m3fn] [--check]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_17059_gb300 as g  # noqa: E402

LAYERS, HEADS, KV_HEADS, DIM, PAGE = 4, 14, 2, 64, 16
VOCAB = 512
PEERS = 4


def csr(seqs):
    off = torch.tensor(np.concatenate([[0], np.cumsum([len(s) for s in seqs])]), dtype=torch.int64, device="cuda")
    return torch.tensor([t for s in seqs for t in s], dtype=torch.int32, device="cuda"), off


def ints(values):
    return torch.tensor(list(values), dtype=torch.int32, device="cuda")


class Model:
    """Queries [n, HEADS, DIM], keys and values [LAYERS, n, KV_HEADS, DIM] of tokens at positions."""

    def __init__(self, dtype, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        table = lambda heads: torch.randn((LAYERS, VOCAB, heads, DIM), device="cuda", generator=gen)  # noqa: E731
        self.tables = dict(q=table(HEADS) * 2, k=table(KV_HEADS), v=table(KV_HEADS))
        self.where = torch.randn((4096, 1, DIM), device="cuda", generator=gen) * 0.5
        self.dtype = dtype

    def rows(self, what, tokens, positions):
        x = self.tables[what][:, tokens.long()]
        return (x + self.where[positions.long() % 4096] if what != "v" else x).to(self.dtype)

    @staticmethod
    def next_token(out):
        return int(out.float().abs().sum(0).argmax()) * 7 % VOCAB


class Node:
    def __init__(self, pages: int, rows: int, dtype):
        self.router = g.Router(PEERS)
        g.p2p_lru_enable(self.router.handle, 0)
        half = torch.float16 if dtype == torch.float16 else torch.bfloat16
        scales = [torch.full((LAYERS, KV_HEADS), 0.02, device="cuda") for _ in "kv"] if dtype == torch.float8_e4m3fn else [None, None]
        self.cache = g.KvCache.empty(LAYERS, pages, PAGE, KV_HEADS, DIM, rows, 64, dtype=dtype, k_scale=scales[0], v_scale=scales[1])
        self.pages, self.model = pages, Model(half)
        self.held = {}                       # row -> the tokens it holds in the cache
        self.free_rows = list(range(rows))
        self.time = 0
        self.hit_tokens = self.prompt_tokens = self.evicted_tokens = 0

    # ---- cache and trie together

    def lru_insert(self, prompts):
        tok, off = csr(prompts)
        self.time += 1
        g.p2p_lru_insert(self.router.handle, 0, tok, tok.numel(), off, len(prompts), self.time)

    def trim(self, keep):
        """Cuts rows down to keep[row] tokens; a row that holds none is free again."""
        if not keep:
            return
        self.cache.trim(ints(keep), ints(keep.values()))
        for row, n in keep.items():
            self.held[row] = self.held[row][:n]
            if n == 0:
                del self.held[row]
                self.free_rows.append(row)

    def make_room(self, pages):
        """Evicts until that many pages and a row are free: least recently used tokens leave the trie, then the rows that held
        them are cut to what the trie still matches of them."""
        while self.held and (not self.free_rows or self.pages - self.cache.stats()["pages_used"] < pages):
            n = g.p2p_lru_evict(self.router.handle, 0, max(pages * PAGE // 2, 1))
            self.evicted_tokens += n
            rows = sorted(self.held)
            tok, off = csr([self.held[r] for r in rows])
            match, _ = self.router.route(tok, off, [0] * PEERS, 0)
            kept = match[:, 0].tolist()
            self.trim({r: k for r, k in zip(rows, kept) if k < len(self.held[r])})
            if n == 0:
                break

    # ---- Algorithm 1 for a batch

    def serve(self, prompts, decode: int, check: bool):
        tok, off = csr(prompts)
        match, peer = self.router.route(tok, off, [0, 40, 50, 60], 1)
        self.router.sync()
        mine = [i for i, p in enumerate(peer.tolist()) if p == 0]
        for i in mine:   # (one after another, so that a request finds what the one before it left)
            self.serve_one(prompts[i], decode, check)
        return len(mine)

    def serve_one(self, prompt, decode, check):
        cache, model = self.cache, self.model
        self.make_room((len(prompt) + decode) // PAGE + 3)
        # The cached sequence that shares most of the prompt; at least the last token is computed anew.
        shared = {r: next((i for i, (a, b) in enumerate(zip(held, prompt)) if a != b), min(len(held), len(prompt)))
                  for r, held in self.held.items()}
        src = max(shared, key=shared.get, default=None)
        n = min(shared.get(src, 0), len(prompt) - 1)
        row = self.free_rows.pop()
        one, tokens = ints([row]), torch.tensor(prompt, dtype=torch.int32, device="cuda")
        if n:
            cache.fork(ints([src]), one, ints([n]))
        cache.extend(one, ints([len(prompt) - n]))
        rest = tokens[n:]
        pos = torch.arange(n, len(prompt), device="cuda")
        cache.write(0, one, torch.tensor([0, len(rest)], device="cuda"), model.rows("k", rest, pos), model.rows("v", rest, pos))
        self.hit_tokens += n
        self.prompt_tokens += len(prompt)
        seq = list(prompt)
        offsets, step = torch.tensor([0, 1], device="cuda"), ints([1])
        for _ in range(decode):
            last = ints([seq[-1]])
            at = torch.tensor([len(seq) - 1], device="cuda")
            q = model.rows("q", last, at)
            outs = [cache.attend(layer, q[layer], seq=one)[0] for layer in range(LAYERS)]
            if check:
                self.check(seq, q, outs)
            seq.append(model.next_token(outs[-1][0]))
            cache.extend(one, step)
            new, at = ints([seq[-1]]), torch.tensor([len(seq) - 1], device="cuda")
            for layer in range(LAYERS):   # (as a model's layers come to them)
                cache.write(layer, one, offsets, model.rows("k", new, at)[layer], model.rows("v", new, at)[layer])
        cache.sync()
        self.held[row] = seq
        self.lru_insert([seq])

    def check(self, seq, q, outs):
        """The layers' attention again, from the tokens alone and without the cache."""
        tokens, pos = torch.tensor(seq, device="cuda"), torch.arange(len(seq), device="cuda")
        eight = self.cache.k_scale is not None
        for layer, out in enumerate(outs):
            k, v = (self.model.rows(w, tokens, pos)[layer].float().repeat_interleave(HEADS // KV_HEADS, 1) for w in "kv")
            x = torch.einsum("hd,thd->ht", q[layer][0].float(), k) * DIM ** -0.5
            want = torch.einsum("ht,thd->hd", torch.softmax(x, 1), v)
            far = float((out[0].float() - want).norm() / want.norm())
            # (16 bits: the result's and the probabilities' rounding; 8 bits: of every key and value, 2^-4 at most.)
            assert far < (0.25 if eight else 0.02), (layer, far)


def run(batches=6, requests=48, decode=4, pages=500, rows=96, dtype=torch.bfloat16, check=False, seed=0):
    rng = np.random.default_rng(seed)
    node = Node(pages, rows, dtype)
    prefixes = [rng.integers(0, VOCAB, int(n)).tolist() for n in rng.integers(60, 400, 12)]
    served = 0
    for _ in range(batches):
        which = np.minimum(rng.zipf(1.5, requests) - 1, len(prefixes) - 1)
        served += node.serve([prefixes[w] + rng.integers(0, VOCAB, int(rng.integers(8, 40))).tolist() for w in which], decode, check)
    before = node.cache.stats()
    node.cache.compact()
    after = node.cache.stats()
    node.cache.sync()
    return dict(served=served, prompt_tokens=node.prompt_tokens, hit_tokens=node.hit_tokens, evicted_tokens=node.evicted_tokens,
                before=before, after=after, launches=node.cache.launch_count())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batches", type=int, default=6)
    ap.add_argument("--requests", type=int, default=48)
    ap.add_argument("--decode", type=int, default=4)
    ap.add_argument("--dtype", default="bfloat16", choices=("bfloat16", "float16", "float8_e4m3fn"))
    ap.add_argument("--check", action="store_true", help="recompute every attention from the tokens alone")
    a = ap.parse_args()
    s = run(a.batches, a.requests, a.decode, dtype=getattr(torch, a.dtype), check=a.check)
    print(f"served {s['served']} requests, {s['hit_tokens']} of {s['prompt_tokens']} prompt tokens from the cache "
          f"({100 * s['hit_tokens'] / max(1, s['prompt_tokens']):.0f}%), {s['evicted_tokens']} tokens evicted")
    print(f"pages in use {s['before']['pages_used']} ({s['before']['pages_shared']} shared), the highest "
          f"{s['before']['pages_end']} before compaction and {s['after']['pages_end']} after")


if __name__ == "__main__":
    main()
