"""The example node: routing, the LRU trie and the paged cache together, every attention recomputed from the tokens."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dtype", ["bfloat16", "float8_e4m3fn"])
def test_serve_node(dtype):
    import serve_node
    s = serve_node.run(batches=4, requests=24, decode=3, pages=260, rows=40, dtype=getattr(torch, dtype), check=True)
    assert s["served"] > 20
    assert 0 < s["hit_tokens"] < s["prompt_tokens"] and s["evicted_tokens"] > 0
    assert s["before"]["pages_shared"] > 0 and s["before"]["pages_used"] <= 260
    assert s["after"]["pages_used"] == s["before"]["pages_used"] == s["after"]["pages_end"]
    assert s["after"]["tokens"] == s["before"]["tokens"]
