"""examples/serve_layers.py with norms of heads, a cache of 8-bit values and shared prefixes: it runs, and what each of them changes is of the size that it should be."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("options", [["--norms"], ["--e4m3"], ["--shared"], ["--norms", "--e4m3", "--shared"]])
def test_the_example_runs(options):
    import serve_layers as S

    stats = S.main(["--layers", "2", "--heads", "8", "--kv-heads", "2", "--dim", "64", "--requests", "5", "--iterations", "4", *options])
    assert stats.pages_used > 0 and stats.seqs == 6


def test_the_same_layers_with_each_option():
    """A prompt, forks of it and their next tokens, through the same weights: prefixes shared change nothing but roundings of sums, 8 bits the outputs by about as much as they
    change keys and values (half a step of 2^-4 at most, 2^-5.5 in the root mean square), a norm all of them."""
    import serve_layers as S

    def outputs(**kw):
        model = S.Layers(2, 8, 2, 64, adapters=2, ranks=(8,), n_pages=120, page_tokens=32, max_seqs=40, **kw)
        try:
            gen = torch.Generator(device="cuda").manual_seed(5)
            x = lambda n: torch.randn(n, model.hidden, generator=gen, device="cuda").bfloat16()  # noqa: E731
            model.cache.add([0])
            got = [model.step(x(700), [0], [0], [700])]
            model.cache.fork(0, np.arange(1, 30))
            for n in (1, 2, 1):
                got.append(model.step(x(29 * n), list(range(1, 30)), [i % 3 - 1 for i in range(1, 30)], [n] * 29))
            assert all(torch.isfinite(y).all() for y in got)
            return torch.cat(got).float()
        finally:
            model.close()

    plain = outputs()
    off = lambda y: float((y - plain).norm() / plain.norm())  # noqa: E731
    assert off(outputs(shared=256)) <= 2.0**-6  # (a few roundings to 8 bits that go the other way in either layer)
    assert 1e-3 < off(outputs(e4m3=True)) <= 5e-2
    assert off(outputs(norms=True)) > 1e-3
    both = outputs(e4m3=True, norms=True, shared=256)
    apart = outputs(e4m3=True, norms=True)
    assert float((both - apart).norm() / apart.norm()) <= 2.0**-6
