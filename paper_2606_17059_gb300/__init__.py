"""GB300 batched routing engine for decentralized, prefix-cache-aware LLM routing.

Thin ctypes binding of ``libp2prouter.so`` (C ABI in ``include/p2p_router.h``).  The functions below
carry the C names and only marshal arguments: every step of routing, matching and tree patching runs in
the library's CUDA kernels.  Device buffers are passed as torch CUDA tensors (or raw integer addresses);
host buffers as numpy arrays.  There is no CPU fallback: importing works without a GPU, but every call
needs the built library and a CUDA device, and raises otherwise.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

from . import build as _build

__all__ = [
    "P2PError", "Router", "KvCache", "build", "library_path",
    "p2p_router_create", "p2p_router_destroy", "p2p_router_set_stream", "p2p_router_sync", "p2p_last_error",
    "p2p_router_num_trees", "p2p_router_launch_count", "p2p_snapshot_build", "p2p_snapshot_view", "p2p_snapshot_free",
    "p2p_flat_tree_validate", "p2p_tree_upload", "p2p_tree_build", "p2p_tree_download", "p2p_tree_apply_delta",
    "p2p_tree_apply_delta_static", "p2p_tree_stats", "p2p_route_batch", "p2p_route_batch_host", "p2p_route_decide",
    "p2p_router_kernel_clock", "p2p_router_kernel_time", "p2p_update_estimates", "p2p_route_batch_decide",
    "p2p_lru_enable", "p2p_lru_insert", "p2p_lru_access", "p2p_lru_evict", "p2p_hit_rate", "p2p_route_prepare",
    "p2p_kv_create", "p2p_kv_destroy", "p2p_kv_set_stream", "p2p_kv_sync", "p2p_kv_last_error", "p2p_kv_launch_count",
    "p2p_kv_stats", "p2p_kv_extend", "p2p_kv_write", "p2p_kv_fork", "p2p_kv_trim", "p2p_kv_compact", "p2p_kv_attend",
]

P2P_OK, P2P_E_INVAL, P2P_E_NOMEM, P2P_E_FORMAT, P2P_E_CUDA, P2P_E_DEVICE = 0, -1, -2, -3, -4, -5
P2P_OP_INSERT, P2P_OP_DELETE = 0, 1
P2P_MEM_HOST, P2P_MEM_DEVICE = 0, 1
P2P_KV_BF16, P2P_KV_F16, P2P_KV_E4M3 = 0, 1, 2
ERROR_NAMES = {-1: "P2P_E_INVAL", -2: "P2P_E_NOMEM", -3: "P2P_E_FORMAT", -4: "P2P_E_CUDA", -5: "P2P_E_DEVICE"}
FLAT_FIELDS = ("label_off", "label_len", "child_begin", "child_count", "term_count",
               "child_first_tok", "child_idx", "labels")

library_path = _build.LIB


def build(force: bool = False) -> str:
    return _build.build(force=force)


class P2PError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {msg}")
        self.code = code


_vp = ctypes.c_void_p
_i32, _i64 = ctypes.c_int32, ctypes.c_int64


class FlatTree(ctypes.Structure):
    _fields_ = [("n_nodes", _i32), ("n_labels", _i32)] + [(f, _vp) for f in FLAT_FIELDS]


class Seqs(ctypes.Structure):
    _fields_ = [("n", _i64), ("seg_begin", _vp), ("seg_off", _vp), ("seg_len", _vp), ("pool", _vp),
                ("n_segs", _i64), ("n_pool", _i64)]


class Delta(ctypes.Structure):
    _fields_ = [("op", _vp), ("seqs", Seqs), ("peer_begin", _vp), ("mem", _i32)]


class KvLayout(ctypes.Structure):
    _fields_ = ([(f, _i32) for f in ("type", "n_layers", "n_pages", "page_tokens", "n_heads", "head_dim", "n_seqs", "max_pages")]
                + [(f, _i64) for f in ("layer_stride", "page_stride", "token_stride", "head_stride")]
                + [(f, _vp) for f in ("k", "v", "k_scale", "v_scale", "table", "length", "refs")])


_lib = None


def _load():
    """Loads the CUDA library (building it first when a source is newer).  Raises if it cannot."""
    global _lib
    if _lib is None:
        path = _build.build()
        if not os.path.exists(path):
            raise RuntimeError(f"CUDA library missing: {path}")
        lib = ctypes.CDLL(path)
        P = ctypes.POINTER
        sig = {
            "p2p_router_create": (ctypes.c_int, [_i32, P(_vp)]),
            "p2p_router_destroy": (None, [_vp]),
            "p2p_router_set_stream": (ctypes.c_int, [_vp, _vp]),
            "p2p_router_sync": (ctypes.c_int, [_vp]),
            "p2p_last_error": (ctypes.c_char_p, [_vp]),
            "p2p_router_num_trees": (_i32, [_vp]),
            "p2p_router_launch_count": (_i64, [_vp]),
            "p2p_snapshot_build": (ctypes.c_int, [P(Seqs), P(_vp)]),
            "p2p_snapshot_view": (None, [_vp, P(FlatTree)]),
            "p2p_snapshot_free": (None, [_vp]),
            "p2p_flat_tree_validate": (ctypes.c_int, [P(FlatTree)]),
            "p2p_tree_upload": (ctypes.c_int, [_vp, _i32, P(FlatTree)]),
            "p2p_tree_build": (ctypes.c_int, [_vp, _i32, P(Seqs)]),
            "p2p_tree_download": (ctypes.c_int, [_vp, _i32, P(_vp)]),
            "p2p_tree_apply_delta": (ctypes.c_int, [_vp, _i32, P(Delta), P(_i64)]),
            "p2p_tree_apply_delta_static": (ctypes.c_int, [_vp, _i32, P(Delta), P(_i64)]),
            "p2p_tree_stats": (ctypes.c_int, [_vp, _i32, P(_i64 * 9)]),
            "p2p_route_batch": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, _i32, _vp, _vp]),
            "p2p_route_batch_host": (ctypes.c_int, [_vp, _vp, _vp, _i64, _vp, _i32, _vp, _vp]),
            "p2p_route_decide": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i32, _vp, _vp, _vp]),
            "p2p_router_kernel_clock": (ctypes.c_int, [_vp, _i32]),
            "p2p_update_estimates": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, P(_i64)]),
            "p2p_route_batch_decide": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, _i32, _vp, _vp, _vp, _vp]),
            "p2p_lru_enable": (ctypes.c_int, [_vp, _i32]),
            "p2p_lru_insert": (ctypes.c_int, [_vp, _i32, _vp, _i64, _vp, _i64, _i64]),
            "p2p_lru_access": (ctypes.c_int, [_vp, _i32, _vp, _i64, _vp, _i64, _i64, _vp]),
            "p2p_lru_evict": (ctypes.c_int, [_vp, _i32, _i64, P(_i64)]),
            "p2p_hit_rate": (ctypes.c_int, [_vp, _vp, _vp, _i64, _vp, _vp]),
            "p2p_route_prepare": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64]),
            "p2p_kv_create": (ctypes.c_int, [P(KvLayout), P(_vp)]),
            "p2p_kv_destroy": (None, [_vp]),
            "p2p_kv_set_stream": (ctypes.c_int, [_vp, _vp]),
            "p2p_kv_sync": (ctypes.c_int, [_vp]),
            "p2p_kv_last_error": (ctypes.c_char_p, [_vp]),
            "p2p_kv_launch_count": (_i64, [_vp]),
            "p2p_kv_stats": (ctypes.c_int, [_vp, P(_i64 * 4)]),
            "p2p_kv_extend": (ctypes.c_int, [_vp, _i32, _vp, _vp]),
            "p2p_kv_write": (ctypes.c_int, [_vp, _i32, _i32, _i32, _vp, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i32]),
            "p2p_kv_fork": (ctypes.c_int, [_vp, _i32, _vp, _vp, _vp]),
            "p2p_kv_trim": (ctypes.c_int, [_vp, _i32, _vp, _vp]),
            "p2p_kv_compact": (ctypes.c_int, [_vp]),
            "p2p_kv_attend": (ctypes.c_int, [_vp, _i32, _i32, _vp, _vp, _i64, _i64, _i32, _i32, ctypes.c_float, _i32, _vp, _i64,
                                             _i64, _vp]),
            "p2p_router_kernel_time": (ctypes.c_int, [_vp, _i32, P(ctypes.c_char_p), P(_i64), P(ctypes.c_double)]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def exported_symbols() -> list[str]:
    """Names of the C entry points this binding declares (all must be exported by the library)."""
    return [n for n in __all__ if n.startswith("p2p_")]


def _check(rc: int, r=None):
    if rc != P2P_OK:
        msg = _load().p2p_last_error(r)
        raise P2PError(rc, msg.decode() if msg else "")


def _addr(x) -> int | None:
    """Address of a torch tensor / numpy array / integer (None stays NULL)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("array must be C-contiguous")
        return x.ctypes.data
    if hasattr(x, "data_ptr"):
        if not x.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return x.data_ptr()
    raise TypeError(f"cannot take the address of {type(x)}")


def _host_i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _load_vec(r, load) -> np.ndarray:
    """The per-tree load as a host int32 array; the library reads one entry per tree."""
    ld = _host_i32(load)
    n = p2p_router_num_trees(r)
    if ld.ndim != 1 or ld.size != n:
        raise ValueError(f"load must have one entry per tree ({n}), got shape {ld.shape}")
    return ld


def _seqs_struct(sl, keep: list) -> Seqs:
    """Seqs struct from an object with seg_begin/seg_off/seg_len/pool (numpy arrays or CUDA tensors)."""
    arrs = []
    for name, dt in (("seg_begin", np.int64), ("seg_off", np.int64), ("seg_len", np.int32), ("pool", np.int32)):
        a = getattr(sl, name)
        if isinstance(a, np.ndarray):
            a = np.ascontiguousarray(a, dtype=dt)
        arrs.append(a)
    keep.extend(arrs)
    sb, so, slen, pool = arrs
    return Seqs(len(sb) - 1, _addr(sb), _addr(so), _addr(slen), _addr(pool), len(so), len(pool))


# ---- the C entry points ---------------------------------------------------------------------------------

def p2p_router_create(P: int):
    h = _vp()
    _check(_load().p2p_router_create(P, ctypes.byref(h)))
    return h


def p2p_router_destroy(r) -> None:
    _load().p2p_router_destroy(r)


def p2p_router_set_stream(r, stream=None) -> None:
    s = None
    if stream is not None:
        s = stream if isinstance(stream, int) else stream.cuda_stream
    _check(_load().p2p_router_set_stream(r, s), r)


def p2p_router_sync(r) -> None:
    _check(_load().p2p_router_sync(r), r)


def p2p_last_error(r=None) -> str:
    m = _load().p2p_last_error(r)
    return m.decode() if m else ""


def p2p_router_num_trees(r) -> int:
    return int(_load().p2p_router_num_trees(r))


def p2p_router_launch_count(r) -> int:
    return int(_load().p2p_router_launch_count(r))


KERNEL_COUNT = 29  # P2P_KERNEL_COUNT: kernels the kernel clock keeps totals for (indices 0 .. 28)


def p2p_router_kernel_clock(r, on: bool) -> None:
    _check(_load().p2p_router_kernel_clock(r, 1 if on else 0), r)


def p2p_router_kernel_time(r, i: int) -> tuple[str, int, float]:
    """(kernel name, timed launches, summed device ms) of kernel i since the clock was switched on."""
    name = ctypes.c_char_p()
    n = _i64()
    ms = ctypes.c_double()
    _check(_load().p2p_router_kernel_time(r, i, ctypes.byref(name), ctypes.byref(n), ctypes.byref(ms)), r)
    return (name.value.decode() if name.value else ""), int(n.value), float(ms.value)


def p2p_snapshot_build(seqlist):
    keep = []
    s = _seqs_struct(seqlist, keep)
    h = _vp()
    _check(_load().p2p_snapshot_build(ctypes.byref(s), ctypes.byref(h)))
    return h


def p2p_snapshot_view(snap) -> dict:
    """Copies a snapshot's arrays into numpy (dict keyed like ``FLAT_FIELDS``)."""
    v = FlatTree()
    _load().p2p_snapshot_view(snap, ctypes.byref(v))
    n, nl = v.n_nodes, v.n_labels
    sizes = {f: n for f in FLAT_FIELDS[:5]}
    sizes.update(child_first_tok=n - 1, child_idx=n - 1, labels=nl)
    out = {}
    for f in FLAT_FIELDS:
        cnt = sizes[f]
        addr = getattr(v, f)
        if cnt == 0 or not addr:
            out[f] = np.zeros(0, np.int32)
        else:
            out[f] = np.ctypeslib.as_array((ctypes.c_int32 * cnt).from_address(addr)).copy()
    return out


def p2p_snapshot_free(snap) -> None:
    _load().p2p_snapshot_free(snap)


def _flat_struct(flat: dict, keep: list) -> FlatTree:
    arrs = {f: _host_i32(flat[f]) for f in FLAT_FIELDS}
    keep.append(arrs)
    t = FlatTree()
    t.n_nodes = len(arrs["label_off"])
    t.n_labels = len(arrs["labels"])
    for f in FLAT_FIELDS:
        setattr(t, f, arrs[f].ctypes.data if len(arrs[f]) else None)
    return t


def p2p_flat_tree_validate(flat: dict) -> int:
    keep = []
    t = _flat_struct(flat, keep)
    return int(_load().p2p_flat_tree_validate(ctypes.byref(t)))


def p2p_tree_upload(r, peer: int, flat: dict) -> None:
    keep = []
    t = _flat_struct(flat, keep)
    _check(_load().p2p_tree_upload(r, peer, ctypes.byref(t)), r)


def p2p_tree_build(r, peer: int, seqlist) -> None:
    keep = []
    s = _seqs_struct(seqlist, keep)
    _check(_load().p2p_tree_build(r, peer, ctypes.byref(s)), r)


def p2p_tree_download(r, peer: int) -> dict:
    h = _vp()
    _check(_load().p2p_tree_download(r, peer, ctypes.byref(h)), r)
    try:
        return p2p_snapshot_view(h)
    finally:
        p2p_snapshot_free(h)


def p2p_tree_apply_delta(r, peer: int, op, seqlist, peer_begin=None, on_device: bool = False) -> int:
    """Applies an ordered INSERT/DELETE delta; returns the number of DELETEs of absent sequences.
    With on_device the op/segment/pool arrays are CUDA tensors, else numpy arrays."""
    keep = []
    if isinstance(op, np.ndarray):
        op = np.ascontiguousarray(op, dtype=np.int32)
    if isinstance(peer_begin, np.ndarray):
        peer_begin = np.ascontiguousarray(peer_begin, dtype=np.int64)
    keep += [op, peer_begin]
    d = Delta(_addr(op), _seqs_struct(seqlist, keep), _addr(peer_begin), P2P_MEM_DEVICE if on_device else P2P_MEM_HOST)
    absent = _i64()
    _check(_load().p2p_tree_apply_delta(r, peer, ctypes.byref(d), ctypes.byref(absent)), r)
    return int(absent.value)


def p2p_tree_apply_delta_static(r, peer: int, op, seqlist, peer_begin=None) -> int:
    """The allocation-free delta call: op/segment/pool arrays (and peer_begin) must be CUDA tensors.
    Returns the number of DELETEs of absent sequences."""
    keep = [op, peer_begin]
    d = Delta(_addr(op), _seqs_struct(seqlist, keep), _addr(peer_begin), P2P_MEM_DEVICE)
    absent = _i64()
    _check(_load().p2p_tree_apply_delta_static(r, peer, ctypes.byref(d), ctypes.byref(absent)), r)
    return int(absent.value)


def p2p_update_estimates(r, tokens, n_tokens: int, offsets, B: int, peer) -> int:
    """Inserts request b into tree peer[b] for every routed request (UpdateTrieEstimate / UpdateTrie of
    Algorithm 1); tokens, offsets and peer are CUDA tensors (or addresses).  Returns the requests inserted."""
    n = _i64()
    _check(_load().p2p_update_estimates(r, _addr(tokens), n_tokens, _addr(offsets), B, _addr(peer), ctypes.byref(n)), r)
    return int(n.value)


def p2p_lru_enable(r, tree: int) -> None:
    _check(_load().p2p_lru_enable(r, tree), r)


def p2p_lru_insert(r, tree: int, tokens, n_tokens: int, offsets, B: int, time: int) -> None:
    """UpdateTrie of a batch at `time` (CUDA tensors tokens/offsets)."""
    _check(_load().p2p_lru_insert(r, tree, _addr(tokens), n_tokens, _addr(offsets), B, time), r)


def p2p_lru_access(r, tree: int, tokens, n_tokens: int, offsets, B: int, time: int, out_match=None) -> None:
    """Requests served at `time`: their matched tokens are touched; out_match (CUDA int32 [B] or None)."""
    _check(_load().p2p_lru_access(r, tree, _addr(tokens), n_tokens, _addr(offsets), B, time, _addr(out_match)), r)


def p2p_lru_evict(r, tree: int, n_tokens: int) -> int:
    """Evicts the n_tokens least recently used leaf tokens; returns how many were evicted."""
    n = _i64()
    _check(_load().p2p_lru_evict(r, tree, n_tokens, ctypes.byref(n)), r)
    return int(n.value)


def p2p_hit_rate(r, match, offsets, B: int, peer, out) -> None:
    """Expected hit rate match[b, peer[b]] / len(b) of routed requests (CUDA tensors; out float32 [B])."""
    _check(_load().p2p_hit_rate(r, _addr(match), _addr(offsets), B, _addr(peer), _addr(out)), r)


STAT_NAMES = ("live_nodes", "node_slots", "child_entries", "label_tokens", "stale_child", "stale_label",
              "cap_node", "cap_child", "cap_label")


def p2p_tree_stats(r, peer: int) -> dict:
    out = (_i64 * 9)()
    _check(_load().p2p_tree_stats(r, peer, ctypes.byref(out)), r)
    return dict(zip(STAT_NAMES, [int(x) for x in out]))


def p2p_route_batch(r, tokens, n_tokens: int, offsets, B: int, load, alpha: int, out_match, out_peer) -> None:
    """Device routing: tokens/offsets/out_match/out_peer are CUDA tensors (or addresses), load is host."""
    ld = _load_vec(r, load)
    _check(_load().p2p_route_batch(r, _addr(tokens), n_tokens, _addr(offsets), B, ld.ctypes.data, alpha,
                                   _addr(out_match), _addr(out_peer)), r)


def _mask(r, excluded, n: int):
    if excluded is None:
        return None
    ex = np.ascontiguousarray(np.asarray(excluded), dtype=np.uint8)
    if ex.size != n:
        raise ValueError(f"excluded must have one entry per tree ({n})")
    return ex


def p2p_route_batch_decide(r, tokens, n_tokens: int, offsets, B: int, load, alpha: int, excluded, out_match, out_peer,
                           out_next=None) -> None:
    """Device routing with excluded trees and the next-best target decided in the walk kernels; tokens, offsets,
    out_match, out_peer and out_next (or None) are CUDA tensors, load and excluded (uint8 per tree, or None)
    host arrays."""
    ld = _load_vec(r, load)
    ex = _mask(r, excluded, ld.size)
    _check(_load().p2p_route_batch_decide(r, _addr(tokens), n_tokens, _addr(offsets), B, ld.ctypes.data, alpha,
                                          ex.ctypes.data if ex is not None else None, _addr(out_match),
                                          _addr(out_peer), _addr(out_next)), r)


def p2p_route_prepare(r, tokens, n_tokens: int, offsets, B: int) -> None:
    """Announces the next batch (CUDA tensors): its grouping overlaps the next delta kernel."""
    _check(_load().p2p_route_prepare(r, _addr(tokens), n_tokens, _addr(offsets), B), r)


def p2p_route_decide(r, match, B: int, load, alpha: int, excluded, out_peer, out_next) -> None:
    """Best and next-best non-excluded tree per request from a device match matrix [B, P] (CUDA tensors or
    addresses); load and excluded (uint8 per tree, or None) are host arrays."""
    ld = _load_vec(r, load)
    n = ld.size
    ex = None
    if excluded is not None:
        ex = np.ascontiguousarray(np.asarray(excluded), dtype=np.uint8)
    if ex is not None and ex.size != n:
        raise ValueError(f"excluded must have one entry per tree ({n})")
    _check(_load().p2p_route_decide(r, _addr(match), B, ld.ctypes.data, alpha,
                                    ex.ctypes.data if ex is not None else None, _addr(out_peer), _addr(out_next)), r)


def p2p_route_batch_host(r, tokens: np.ndarray, offsets: np.ndarray, B: int, load, alpha: int,
                         out_match: np.ndarray, out_peer: np.ndarray) -> None:
    """Host routing: every array is a host numpy array (pinned memory copies faster)."""
    ld = _load_vec(r, load)
    for a, dt in ((tokens, np.int32), (offsets, np.int64), (out_match, np.int32), (out_peer, np.int32)):
        if not isinstance(a, np.ndarray) or a.dtype != dt or not a.flags["C_CONTIGUOUS"]:
            raise TypeError("host routing needs C-contiguous numpy arrays (int32 tokens/outputs, int64 offsets)")
    if B > 0 and (offsets.size < B + 1 or out_match.size < B * ld.size or out_peer.size < B
                  or tokens.size < int(offsets[B])):
        raise ValueError("host routing arrays are smaller than B requests need")
    _check(_load().p2p_route_batch_host(r, _addr(tokens), _addr(offsets), B, ld.ctypes.data, alpha,
                                        _addr(out_match), _addr(out_peer)), r)


# ---- the paged key-value cache ----------------------------------------------------------------------------

def _kv_check(rc: int, kv=None):
    if rc != P2P_OK:
        msg = _load().p2p_kv_last_error(kv)
        raise P2PError(rc, msg.decode() if msg else "")


def p2p_kv_create(layout: KvLayout):
    """Handle on the cache that `layout` describes (its device arrays must outlive the handle)."""
    h = _vp()
    _kv_check(_load().p2p_kv_create(ctypes.byref(layout), ctypes.byref(h)))
    h.stream, h.stream_address = None, 0  # (the calls' stream, for KvCache: as p2p_kv_set_stream was last given it)
    return h


def p2p_kv_destroy(kv) -> None:
    _load().p2p_kv_destroy(kv)


def p2p_kv_set_stream(kv, stream=None) -> None:
    s = None
    if stream is not None:
        s = stream if isinstance(stream, int) else stream.cuda_stream
    _kv_check(_load().p2p_kv_set_stream(kv, s), kv)
    if isinstance(kv, _vp):
        kv.stream, kv.stream_address = stream, s or 0


def p2p_kv_sync(kv) -> None:
    _kv_check(_load().p2p_kv_sync(kv), kv)


def p2p_kv_last_error(kv=None) -> str:
    m = _load().p2p_kv_last_error(kv)
    return m.decode() if m else ""


def p2p_kv_launch_count(kv) -> int:
    return int(_load().p2p_kv_launch_count(kv))


KV_STAT_NAMES = ("pages_used", "pages_shared", "pages_end", "tokens")


def p2p_kv_stats(kv) -> dict:
    out = (_i64 * 4)()
    _kv_check(_load().p2p_kv_stats(kv, ctypes.byref(out)), kv)
    return dict(zip(KV_STAT_NAMES, [int(x) for x in out]))


def p2p_kv_extend(kv, n: int, seq, count) -> None:
    """Room for count[i] more tokens of sequence seq[i] (CUDA int32 tensors or addresses, as below)."""
    _kv_check(_load().p2p_kv_extend(kv, n, _addr(seq), _addr(count)), kv)


def p2p_kv_write(kv, layer: int, n_layers: int, n: int, seq, offsets, n_tokens: int, k, v, layer_stride: int, token_stride: int,
                 head_stride: int, dtype: int) -> None:
    """Keys and values of the sequences' last tokens; k and v are addresses (their strides are arguments)."""
    _kv_check(_load().p2p_kv_write(kv, layer, n_layers, n, _addr(seq), _addr(offsets), n_tokens, k, v, layer_stride, token_stride,
                                   head_stride, dtype), kv)


def p2p_kv_fork(kv, n: int, src, dst, n_tokens) -> None:
    _kv_check(_load().p2p_kv_fork(kv, n, _addr(src), _addr(dst), _addr(n_tokens)), kv)


def p2p_kv_trim(kv, n: int, seq, n_tokens) -> None:
    _kv_check(_load().p2p_kv_trim(kv, n, _addr(seq), _addr(n_tokens)), kv)


def p2p_kv_compact(kv) -> None:
    _kv_check(_load().p2p_kv_compact(kv), kv)


def p2p_kv_attend(kv, layer: int, n: int, seq, q, q_row_stride: int, q_head_stride: int, dtype: int, n_heads: int, scale: float,
                  window: int, out, out_row_stride: int, out_head_stride: int, lse=None) -> None:
    """One new token of each sequence; q and out are addresses (their strides are arguments)."""
    _kv_check(_load().p2p_kv_attend(kv, layer, n, _addr(seq), q, q_row_stride, q_head_stride, dtype, n_heads, scale, window, out,
                                    out_row_stride, out_head_stride, _addr(lse)), kv)


# ---- convenience wrappers ---------------------------------------------------------------------------------

class KvCache:
    """A paged key-value cache (p2p_kv) over the caller's CUDA tensors.

    k, v      [layers, pages, tokens a page, heads, head dim] of bfloat16, float16 or float8_e4m3fn, strided alike; the
              order of the dimensions in memory is free (see p2p_kv_layout), the last is contiguous
    table     int32 [sequences, pages a sequence]; length int32 [sequences]; refs int32 [pages]
    k_scale, v_scale   float32 [layers, heads], with float8_e4m3fn only

    ``KvCache.empty`` allocates them.  Calls run on `stream` (torch's current one at construction; ``set_stream`` gives them
    another) and return before their work is done; tensors made or used on another stream are the caller's to order.  What
    ``attend`` allocates itself is allocated on the calls' stream: a program on another one waits for that stream before it
    reads the result, and keeps it (or calls its record_stream) until that is done.  A CUDA graph records the calls of a cache
    whose stream is the one being captured.  No call records gradients.  What the device finds wrong is raised by ``sync``."""

    def __init__(self, k, v, table, length, refs, k_scale=None, v_scale=None, stream=None):
        import torch
        self._types = {torch.bfloat16: P2P_KV_BF16, torch.float16: P2P_KV_F16, torch.float8_e4m3fn: P2P_KV_E4M3}
        if k.dim() != 5 or k.dtype not in self._types or v.dtype != k.dtype or v.shape != k.shape or v.stride() != k.stride():
            raise ValueError("k and v must be [layers, pages, page tokens, heads, head dim] of one type and of the same strides")
        if k.shape[4] > 1 and k.stride(4) != 1:
            raise ValueError("the last dimension of k and v must be contiguous")
        layers, pages, page, heads, dim = k.shape
        if table.dim() != 2 or tuple(length.shape) != (table.shape[0],) or tuple(refs.shape) != (pages,):
            raise ValueError("table must be [sequences, entries], length [sequences], refs [pages]")
        scales = (k_scale, v_scale)
        for t in scales:
            if t is not None and tuple(t.shape) != (layers, heads):
                raise ValueError("scales must be [layers, heads]")
        for t, dtype in ((table, torch.int32), (length, torch.int32), (refs, torch.int32), (k_scale, torch.float32),
                         (v_scale, torch.float32)):
            if t is not None and (t.dtype != dtype or not t.is_contiguous()):
                raise ValueError(f"table, length, refs (int32) and scales (float32) must be contiguous: got {t.dtype}")
        if any(t is not None and t.device != k.device for t in (v, table, length, refs, *scales)) or not k.is_cuda:
            raise ValueError("the cache's tensors must be on one CUDA device")
        self.k, self.v, self.table, self.length, self.refs = k, v, table, length, refs
        self.k_scale, self.v_scale = scales
        self.layers, self.heads, self.dim, self.n_seqs = layers, heads, dim, table.shape[0]
        self._int32, self._int64, self._float32, self._empty = torch.int32, torch.int64, torch.float32, torch.empty
        lib = _load()  # (the calls of a decode step go to the library's functions directly)
        self._extend, self._trim, self._fork, self._write, self._attend = (
            lib.p2p_kv_extend, lib.p2p_kv_trim, lib.p2p_kv_fork, lib.p2p_kv_write, lib.p2p_kv_attend)
        a = KvLayout(self._types[k.dtype], layers, pages, page, heads, dim, table.shape[0], table.shape[1], *k.stride()[:4],
                     k.data_ptr(), v.data_ptr(), _addr(k_scale), _addr(v_scale), table.data_ptr(), length.data_ptr(), refs.data_ptr())
        self.device, self._index = k.device, k.device.index
        self._cuda, self._current = torch.cuda, torch._C._cuda_getCurrentRawStream
        with torch.cuda.device(k.device):
            self._h = p2p_kv_create(a)
            if stream is None:
                stream = torch.cuda.current_stream()
        p2p_kv_set_stream(self._h, stream)

    @classmethod
    def empty(cls, layers: int, pages: int, page: int, heads: int, dim: int, n_seqs: int, max_pages: int, dtype=None, k_scale=None,
              v_scale=None, device="cuda", stream=None):
        """An empty cache whose pages keep each head's tokens together (dtype: bfloat16 unless given)."""
        import torch
        k, v = (torch.zeros((layers, pages, heads, page, dim), dtype=dtype or torch.bfloat16, device=device).transpose(2, 3)
                for _ in "kv")
        table, length, refs = (torch.zeros(s, dtype=torch.int32, device=device) for s in ((n_seqs, max_pages), n_seqs, pages))
        return cls(k, v, table, length, refs, k_scale, v_scale, stream)

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            p2p_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    @property
    def stream(self):
        """The calls' stream."""
        return None if self._h is None else self._h.stream

    def set_stream(self, stream) -> None:
        """Gives the calls another stream (waits for the work queued on the one before)."""
        p2p_kv_set_stream(self._h, stream)

    def _empty_on_stream(self, shape, dtype, device):
        """torch.empty, where torch's current stream is not the calls'."""
        s = self._h.stream
        if s is None or isinstance(s, int):
            s = self._cuda.ExternalStream(s, device) if s else self._cuda.default_stream(device)
        with self._cuda.stream(s):
            return self._empty(shape, dtype=dtype, device=device)

    def _list(self, t, n: int, dtype) -> int:
        """Address of a list of n entries."""
        if t.dtype is not dtype or t.numel() != n or t.device != self.device or not t.is_contiguous():
            raise ValueError(f"lists must be contiguous {dtype} tensors on the cache's device, here of {n} entries")
        return t.data_ptr()

    def extend(self, seq, count) -> None:
        """Room for count[i] more tokens of sequence seq[i]; shared last pages are copied first."""
        n, i32 = seq.numel(), self._int32
        rc = self._extend(self._h, n, self._list(seq, n, i32), self._list(count, n, i32))
        if rc:
            _kv_check(rc, self._h)

    def trim(self, seq, n_tokens) -> None:
        """Sequence seq[i] keeps its first n_tokens[i] tokens."""
        n, i32 = seq.numel(), self._int32
        rc = self._trim(self._h, n, self._list(seq, n, i32), self._list(n_tokens, n, i32))
        if rc:
            _kv_check(rc, self._h)

    def fork(self, src, dst, n_tokens) -> None:
        """The empty sequence dst[i] becomes the first n_tokens[i] tokens of src[i], whose pages it shares."""
        n, i32 = src.numel(), self._int32
        rc = self._fork(self._h, n, self._list(src, n, i32), self._list(dst, n, i32), self._list(n_tokens, n, i32))
        if rc:
            _kv_check(rc, self._h)

    def compact(self) -> None:
        """Moves the pages in use to the front of the pool."""
        p2p_kv_compact(self._h)

    def write(self, layer: int, seq, offsets, k, v) -> None:
        """Keys and values of the last offsets[i+1] - offsets[i] tokens of sequence seq[i]: k and v [layers, tokens, heads,
        head dim] for layers layer, layer + 1, ... (or [tokens, heads, head dim] for one); offsets int64 [n + 1]."""
        n, shape, strides, kind = seq.numel(), k.shape, k.stride(), self._types.get(k.dtype)
        if len(shape) == 3:
            shape, strides = (1, *shape), (0, *strides)
        if (len(shape) != 4 or shape[2] != self.heads or shape[3] != self.dim or kind is None or v.dtype is not k.dtype
                or v.shape != k.shape or v.stride() != k.stride() or (self.dim > 1 and strides[3] != 1)):
            raise ValueError("k and v must be [layers, tokens, heads, head dim] or [tokens, heads, head dim], strided alike, "
                             "the last dimension contiguous")
        if k.device != self.device or v.device != self.device:
            raise ValueError("tensors must be on the cache's device")
        if not 0 <= layer <= self.layers:
            layer = -1  # (refused by the call, whose numbers are of 32 bits)
        rc = self._write(self._h, layer, shape[0], n, self._list(seq, n, self._int32), self._list(offsets, n + 1, self._int64),
                         shape[1], k.data_ptr(), v.data_ptr(), strides[0], strides[1], strides[2], kind)
        if rc:
            _kv_check(rc, self._h)

    def attend(self, layer: int, q, scale=None, seq=None, window: int = 0, out=None, lse=None):
        """One new token of each sequence (of seq, int32, or sequences 0, 1, ...): q [n, query heads, head dim]; scale: head
        dim ** -0.5 unless given.  Returns (out like q, lse float32 [n, query heads])."""
        shape, dtype = q.shape, q.dtype
        n, heads, dim = shape
        row, head, inner = q.stride()
        kind = self._types.get(dtype)
        if dim != self.dim or kind is None or inner != 1 and dim > 1 or q.device != self.device:
            raise ValueError("q must be [n, query heads, head dim] on the cache's device, the last dimension contiguous")
        empty = self._empty if self._current(self._index) == self._h.stream_address else self._empty_on_stream
        if out is None:
            out = empty(shape, dtype=dtype, device=self.device)
            out_row, out_head = heads * dim, dim
        else:
            if out.shape != shape or out.dtype is not dtype or out.device != self.device or out.stride(2) != 1 and dim > 1:
                raise ValueError("out must be like q, the last dimension contiguous")
            out_row, out_head, _ = out.stride()
        if lse is None:
            lse = empty((n, heads), dtype=self._float32, device=self.device)
        elif (tuple(lse.shape) != (n, heads) or lse.dtype is not self._float32 or lse.device != self.device
              or not lse.is_contiguous()):
            raise ValueError("lse must be contiguous float32 [n, query heads]")
        if not 0 <= layer < self.layers:
            layer = -1  # (refused by the call, whose numbers are of 32 bits, as is a negative window)
        if not 0 <= window < 1 << 31:
            window = -1 if window < 0 else (1 << 31) - 1
        rc = self._attend(self._h, layer, n, None if seq is None else self._list(seq, n, self._int32), q.data_ptr(), row, head, kind,
                          heads, dim ** -0.5 if scale is None else scale, window, out.data_ptr(), out_row, out_head, lse.data_ptr())
        if rc:
            _kv_check(rc, self._h)
        return out, lse

    def stats(self) -> dict:
        """Pages in use, shared pages, the highest page in use + 1, tokens held (waits for queued work)."""
        return p2p_kv_stats(self._h)

    def launch_count(self) -> int:
        return p2p_kv_launch_count(self._h)

    def sync(self) -> None:
        """Waits for queued work; raises what the device found wrong since the last call."""
        p2p_kv_sync(self._h)


class Router:
    """Owns one p2p_router.  Device work runs on torch's current CUDA stream at construction."""

    def __init__(self, P: int, stream=None):
        import torch
        self.P = P
        self._h = p2p_router_create(P)
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        p2p_router_set_stream(self._h, self.stream)

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None:
            p2p_router_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    def build(self, peer: int, seqlist) -> None:
        p2p_tree_build(self._h, peer, seqlist)

    def upload(self, peer: int, flat: dict) -> None:
        p2p_tree_upload(self._h, peer, flat)

    def download(self, peer: int) -> dict:
        return p2p_tree_download(self._h, peer)

    def stats(self, peer: int) -> dict:
        return p2p_tree_stats(self._h, peer)

    def apply_delta(self, peer: int, op, seqlist, peer_begin=None, on_device: bool = False) -> int:
        return p2p_tree_apply_delta(self._h, peer, op, seqlist, peer_begin, on_device)

    def sync(self) -> None:
        p2p_router_sync(self._h)

    def update_estimates(self, tokens, offsets, peer) -> int:
        """After routing: request b (CUDA tensors tokens/offsets) goes into tree peer[b]; returns the count."""
        return p2p_update_estimates(self._h, tokens, tokens.numel(), offsets, offsets.numel() - 1, peer)

    def launch_count(self) -> int:
        return p2p_router_launch_count(self._h)

    def kernel_clock(self, on: bool) -> None:
        p2p_router_kernel_clock(self._h, on)

    def kernel_times(self) -> dict:
        """{kernel name: (launches, summed device ms)} of the kernels launched since the clock was switched on."""
        out = {}
        for i in range(KERNEL_COUNT):
            name, n, ms = p2p_router_kernel_time(self._h, i)
            if n:
                out[name] = (n, ms)
        return out

    def route(self, tokens, offsets, load, alpha: int, out_match=None, out_peer=None):
        """tokens (int32) and offsets (int64) are CUDA tensors; returns (match [B,P], peer [B]) tensors."""
        import torch
        B = offsets.numel() - 1
        if out_match is None:
            out_match = torch.empty((B, self.P), dtype=torch.int32, device=tokens.device)
        if out_peer is None:
            out_peer = torch.empty(B, dtype=torch.int32, device=tokens.device)
        p2p_route_batch(self._h, tokens, tokens.numel(), offsets, B, load, alpha, out_match, out_peer)
        return out_match, out_peer

    def route_decide(self, tokens, offsets, load, alpha: int, excluded=None, want_next: bool = True):
        """Routing with excluded trees and the next-best target in one pass; returns (match [B,P], peer [B],
        next [B] or None) CUDA tensors."""
        import torch
        B = offsets.numel() - 1
        m = torch.empty((B, self.P), dtype=torch.int32, device=tokens.device)
        p = torch.empty(B, dtype=torch.int32, device=tokens.device)
        n = torch.empty(B, dtype=torch.int32, device=tokens.device) if want_next else None
        p2p_route_batch_decide(self._h, tokens, tokens.numel(), offsets, B, load, alpha, excluded, m, p, n)
        return m, p, n

    def decide(self, match, load, alpha: int, excluded=None, out_peer=None, out_next=None):
        """match is a CUDA int32 tensor [B, P]; returns (peer [B], next [B]) CUDA tensors."""
        import torch
        B = match.shape[0]
        if out_peer is None:
            out_peer = torch.empty(B, dtype=torch.int32, device=match.device)
        if out_next is None:
            out_next = torch.empty(B, dtype=torch.int32, device=match.device)
        p2p_route_decide(self._h, match, B, load, alpha, excluded, out_peer, out_next)
        return out_peer, out_next

    def route_host(self, tokens: np.ndarray, offsets: np.ndarray, load, alpha: int, out_match=None, out_peer=None):
        B = len(offsets) - 1
        if out_match is None:
            out_match = np.empty((B, self.P), np.int32)
        if out_peer is None:
            out_peer = np.empty(B, np.int32)
        p2p_route_batch_host(self._h, tokens, offsets, B, load, alpha, out_match, out_peer)
        return out_match, out_peer
