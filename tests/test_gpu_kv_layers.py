"""The adapter cache and the key-value cache together, as examples/serve_layers.py runs them: two layers with adapters over
iterations of prompts and single tokens, with forks, ends and moved pages, against the same layers computed token by token in plain torch."""
import math
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


class Plain:
    """One request's layers in fp32 with the roundings to bf16 that the served path stores: projections, turned keys and queries, outputs."""

    def __init__(self, model):
        self.m, self.k, self.v = model, [], []

    def copy(self):
        c = Plain(self.m)
        c.k, c.v = [t.clone() for t in self.k], [t.clone() for t in self.v]
        return c

    def step(self, x, adapter, weights):
        m = self.m
        b = lambda t: t.bfloat16().float()  # noqa: E731
        x = x.float()

        def project(layer, p, x):
            y = b(x @ m.w[layer][p].float())
            if adapter >= 0:
                A, Bm = weights[adapter][layer][p]
                y = b(y + (x @ A) @ Bm)
            return y

        def turn(t, first):
            c, s = m.rope[first : first + len(t), None].chunk(2, -1)
            u, w = t.chunk(2, -1)
            return b(torch.cat([u * c - w * s, w * c + u * s], -1))

        for layer in range(len(m.w)):
            n, first = len(x), len(self.k[layer]) if len(self.k) > layer else 0
            q, k, v = (project(layer, p, x) for p in range(3))
            q, k, v = turn(q.view(n, m.heads, m.dim), first), turn(k.view(n, m.kv_heads, m.dim), first), v.view(n, m.kv_heads, m.dim)
            if len(self.k) <= layer:
                self.k.append(k), self.v.append(v)
            else:
                self.k[layer], self.v[layer] = torch.cat([self.k[layer], k]), torch.cat([self.v[layer], v])
            keys, vals = self.k[layer].repeat_interleave(m.heads // m.kv_heads, 1), self.v[layer].repeat_interleave(m.heads // m.kv_heads, 1)
            out = torch.empty(n, m.heads, m.dim, device="cuda")
            for h in range(m.heads):
                s = q[:, h] @ keys[:, h].T.contiguous() / math.sqrt(m.dim)
                s = s.masked_fill(torch.arange(s.shape[1], device="cuda") > first + torch.arange(n, device="cuda")[:, None], float("-inf"))
                out[:, h] = torch.softmax(s, -1) @ vals[:, h].contiguous()
            y = project(layer, 3, b(out.view(n, -1)))
            x = b(torch.nn.functional.layer_norm(b(x + y), (m.hidden,)))
        return x


def test_served_layers_match_plain_ones():
    import serve_layers as S

    rng = np.random.default_rng(0)
    model = S.Layers(2, 8, 2, 64, adapters=3, ranks=(8, 32), n_pages=60, page_tokens=32, max_seqs=16)
    try:
        # the adapters as fill() got them (the example draws them from this generator in this order)
        rw = np.random.default_rng(0)
        weights = []
        for a in range(3):
            r = model.rank[a]
            weights.append([[tuple(torch.from_numpy(rw.normal(0, 0.05, s).astype(np.float32)).bfloat16().float().cuda() for s in ((i, r), (r, o))) for i, o in model.projs] for _ in range(2)])
        plain, adapter = {i: Plain(model) for i in range(5)}, {0: 0, 1: -1, 2: 1, 3: 2, 4: 0}
        model.cache.add(list(plain))
        lengths = {0: 40, 1: 1, 2: 70, 3: 7, 4: 33}
        gen = torch.Generator(device="cuda").manual_seed(3)
        for it in range(7):
            if it == 3:
                model.cache.fork(0, [10, 11])
                for i in (10, 11):
                    plain[i], adapter[i], lengths[i] = plain[0].copy(), adapter[0], 1
                model.cache.free([2, 3])
                for i in (2, 3):
                    del plain[i], lengths[i]
                assert model.cache.compact() > 0
                model.cache.set_limit(model.cache.stats().pages_end + 8)
            ids = list(lengths)
            x = torch.randn(sum(lengths.values()), model.hidden, generator=gen, device="cuda").bfloat16()
            y = model.step(x, ids, [adapter[i] for i in ids], [lengths[i] for i in ids]).float()
            at = 0
            for i in ids:
                want = plain[i].step(x[at : at + lengths[i]], adapter[i], weights)
                err = (y[at : at + lengths[i]] - want).norm() / want.norm()
                # each of the two layers rounds a dozen times to 8 bits, differently where sums are formed in another order: 2^-8 times a few
                assert float(err) <= 3e-2, (it, i, float(err))
                at += lengths[i]
            lengths = {i: (1 if rng.random() < 0.7 else int(rng.integers(2, 30))) for i in ids}
        assert model.cache.stats().pages_copied > 0
    finally:
        model.close()


def test_the_example_runs():
    import serve_layers as S

    stats = S.main(["--layers", "2", "--heads", "8", "--kv-heads", "2", "--dim", "64", "--requests", "5", "--iterations", "4"])
    assert stats.pages_used > 0 and stats.seqs == 6


def test_the_example_runs_with_many_requests():
    import serve_layers as S

    stats = S.main(["--layers", "1", "--heads", "4", "--kv-heads", "2", "--dim", "64", "--requests", "70", "--iterations", "3"])
    assert stats.seqs == 38
