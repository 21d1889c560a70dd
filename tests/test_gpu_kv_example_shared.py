"""examples/serve_layers.py --shared: the continuations of a request share its pages, and attention reads them once."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("sizes", [[], ["--heads", "8", "--kv-heads", "2", "--dim", "64", "--requests", "5", "--iterations", "4", "--e4m3", "--norms"]])
@pytest.mark.parametrize("option,shares", [([], False), (["--shared"], True), (["--shared", "32"], True), (["--shared", "100000"], False)])
def test_what_the_example_shares(sizes, option, shares, monkeypatch):
    import serve_layers as S
    from paper_2411_17741_amd import binding as B

    made, seen = S.KvCache.batch, []

    def batch(self, *a, **kw):
        b = made(self, *a, **kw)
        seen.append(B.lora_kv_batch_prefixes(b)[1].n_segments)
        return b

    monkeypatch.setattr(S.KvCache, "batch", batch)
    S.main(["--layers", "2", *sizes, *option])
    half = len(seen) // 2  # request 0 and three continuations, from there on
    assert set(seen[:half]) == {0} and set(seen[half:]) == ({4} if shares else {0})
