"""The paged cache's calls on streams: which one the results belong to, and a change of it."""
import pytest

import paper_2606_17059_gb300 as g

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from test_gpu_kv_attend import make, query


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
