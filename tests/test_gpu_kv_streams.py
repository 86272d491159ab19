"""The paged cache's calls on streams: which one the results belong to, a change of it, handles made after others, and what
handles and calls allocate."""
import os
import subprocess
import sys

import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

if torch.cuda.is_available():
    from test_gpu_kv_attend import check, make, query


def test_results_belong_to_the_calls_stream():
    """On another stream there is memory that was given back while its last use is still queued: no result lies there."""
    c = make([100, 9000, 5], 2, 64, 16, "bf16")
    q = query(3, 14, 64, torch.bfloat16)
    want, want_lse = c.attend(0, q)
    c.sync()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        for like in (want, want_lse):
            torch.empty_like(like)             # (the pool of this stream has blocks of both sizes)
        torch.cuda._sleep(20_000_000)          # 10 ms
        used = [torch.full_like(want, 7.0), torch.full_like(want_lse, 7.0)]
        del used
        out, lse = c.attend(0, q)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_the_stream_is_changed():
    c = make([100, 9000, 5], 2, 64, 16, "bf16")
    q = query(3, 14, 64, torch.bfloat16)
    want, want_lse = c.attend(0, q)
    c.sync()
    assert c.stream == torch.cuda.current_stream()
    st = torch.cuda.Stream()
    for stream in (st, st.cuda_stream):        # (an address will do)
        c.set_stream(stream)
        assert c.stream == stream
        with torch.cuda.stream(st):
            out, lse = c.attend(0, q)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                again, again_lse = c.attend(0, q)
            graph.replay()
            st.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert torch.equal(again, want) and torch.equal(again_lse, want_lse)
    out, lse = c.attend(0, q)                  # (from the default stream, on st)
    c.sync()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    g.p2p_kv_set_stream(c.handle, None)
    assert c.stream is None
    with torch.cuda.stream(st):
        out, lse = c.attend(0, q)
    c.sync()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    c.close()
    assert c.stream is None


def test_handles_after_handles():
    """Scratch that a destroyed handle gave back is a later one's, whose calls find in it what a new one's would."""
    st = torch.cuda.Stream()
    for turn in range(6):
        lengths = [[70001], [40, 0, 300], [5] * 2000][turn % 3]
        c = make(lengths, 4, 128, 16, "bf16", seed=turn)
        torch.cuda.synchronize()
        if turn % 2:
            c.set_stream(st)
        q = query(len(lengths), 8, 128, torch.bfloat16, seed=turn)
        got = c.attend(0, q)
        c.sync()
        check(c, 0, q, 128 ** -0.5, got)
        if turn != 3:
            c.close()                          # (with nothing queued; the others are closed with a call under way)
        else:
            c.attend(0, q)
            c.close()
            c.close()


def test_calls_allocate_nothing():
    """Once a handle is made, calls take no device memory from the driver, nor from torch beyond attend's own results."""
    c = make([100, 9000, 5], 2, 64, 16, "bf16", spare=40)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q = query(3, 14, 64, torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty((3, 14), device="cuda")
    k = torch.zeros((1, 7, 2, 64), device="cuda", dtype=torch.bfloat16)
    seq, other, count, less, off = i32(0), i32(2), i32(7), i32(90), torch.tensor([0, 7], device="cuda")
    none, part = i32(0), i32(33)

    def calls():
        c.extend(seq, count)
        c.write(0, seq, off, k, k)
        c.attend(0, q, out=out, lse=lse)
        c.trim(other, none)
        c.fork(seq, other, part)
        c.extend(other, count)
        c.compact()
        c.trim(seq, less)
        c.sync()

    c.trim(seq, less)
    calls()
    torch.cuda.synchronize()
    free, held = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(20):
        calls()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free
    assert torch.cuda.memory_stats()["allocation.all.allocated"] == held


def test_scratch_is_what_the_kernels_need():
    """Of a handle's scratch the kernels for one size of rows use all; in a process of its own, as scratch is kept."""
    code = """
import torch, paper_2606_17059_gb300 as g
first = g.KvCache.empty(1, 4, 16, 1, 16, 1, 1)     # (the library's kernels and its pool are there)
torch.cuda.synchronize()
made, free = [], torch.cuda.mem_get_info()[0]
for _ in range(8):
    made.append(g.KvCache.empty(1, 4, 16, 4, 256, 1, 1))
torch.cuda.synchronize()
print((free - torch.cuda.mem_get_info()[0]) / 8e6)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0, r.stderr
    assert float(r.stdout) < 46, r.stdout      # 40.2 MB of parts; the driver gives memory in blocks
