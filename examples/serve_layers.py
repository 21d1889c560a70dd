"""Serving a few layers of a model with adapters: what an iteration does with the adapter cache and the key-value cache together.

    python examples/serve_layers.py [--layers 2] [--heads 32] [--kv-heads 8] [--dim 128] [--requests 8] [--iterations 6]

Every iteration forms a batch -- the prompts of new requests, one token of each running one -- and runs, per layer, the q, k, v
projections with the adapters of the requests, lora_kv_append (positions, keys and values into the pages), lora_kv_attend and the o projection with
its adapters.  Half way one request is forked into continuations that share its pages, some requests end, and the pages in use
are moved together so that the rest of the memory is free for adapters.  The model is synthetic (random weights, no MLP); the
base projections are plain matrix products."""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_17741_amd import KvCache, LoraPool  # noqa: E402
from paper_2411_17741_amd import binding as B  # noqa: E402


def rope_table(positions: int, dim: int) -> torch.Tensor:
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float().cuda()


class Layers:
    """Weights of the layers, adapters in their pool, keys and values in their cache."""

    def __init__(self, layers, heads, kv_heads, dim, adapters, ranks=(8, 32), max_tokens=4096, max_seqs=64, n_pages=512, page_tokens=64, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *shape: (torch.randn(*shape, generator=gen, device="cuda") * shape[0] ** -0.5).bfloat16()  # noqa: E731
        self.hidden, self.heads, self.kv_heads, self.dim = heads * dim, heads, kv_heads, dim
        widths = [heads * dim, kv_heads * dim, kv_heads * dim]
        self.projs = [(self.hidden, w) for w in widths] + [(heads * dim, self.hidden)]
        self.w = [[rnd(i, o) for i, o in self.projs] for _ in range(layers)]
        self.pool = LoraPool(self.projs, layers, sorted(set(ranks)), [adapters] * len(set(ranks)), B.LORA_BF16, max_tokens=max_tokens, max_segments=max_seqs)
        self.slot, self.rank = [], []
        rng = np.random.default_rng(seed)
        for a in range(adapters):
            rank = int(ranks[a % len(ranks)])
            self.slot.append(sorted(set(ranks)).index(rank) * adapters + a)
            self.rank.append(rank)
            for layer in range(layers):
                for p, (i, o) in enumerate(self.projs):
                    self.pool.fill(self.slot[a], a, rank, 1.0, layer, p, rng.normal(0, 0.05, (i, rank)).astype(np.float32), rng.normal(0, 0.05, (rank, o)).astype(np.float32))
        torch.cuda.synchronize()
        self.pool.fills_done()
        self.cache = KvCache(layers, heads, kv_heads, dim, n_pages, page_tokens=page_tokens, max_seqs=max_seqs, max_batch_seqs=max_seqs, max_batch_tokens=max_tokens)
        self.rope = rope_table(8192, dim)

    def step(self, x, requests, adapters, lengths):
        """x [T][hidden], the packed tokens of `requests` (lengths[i] of request i, adapter adapters[i] or -1) -> the layers' output"""
        off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        slots = np.asarray([self.slot[a] if a >= 0 else -1 for a in adapters], np.int32)
        ranks = np.asarray([self.rank[a] if a >= 0 else 0 for a in adapters], np.int32)
        plan = self.pool.plan(len(x), off, slots, ranks)
        batch = self.cache.batch(np.asarray(requests, np.int64), off)
        scale = 1.0 / math.sqrt(self.dim)
        for layer, w in enumerate(self.w):
            q, k, v = (x @ w[p] for p in range(3))
            for p, y in enumerate((q, k, v)):
                self.pool.apply_plan(plan, layer, p, x, y, 1.0)
            self.cache.append(batch, layer, k, v, q=q, rope=self.rope)  # q turns in place
            out = torch.empty_like(q)
            self.cache.attend(batch, layer, q, out, scale)
            y = out @ w[3]
            self.pool.apply_plan(plan, layer, 3, out, y, 1.0)
            x = torch.nn.functional.layer_norm((x + y).float(), (self.hidden,)).bfloat16()
        self.pool.plan_destroy(plan)
        self.cache.batch_destroy(batch)
        return x

    def close(self):
        self.cache.close()
        self.pool.close()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 2), ("heads", 32), ("kv-heads", 8), ("dim", 128), ("requests", 8), ("iterations", 6)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    rng = np.random.default_rng(1)
    # room for prompts of up to 300 tokens, a token in each iteration after that, and the continuations
    seqs, each = a.requests + 3, 300 + a.iterations
    model = Layers(a.layers, a.heads, a.kv_heads, a.dim, adapters=4, max_tokens=max(4096, 300 * seqs), max_seqs=max(64, seqs), n_pages=max(512, seqs * (each // 64 + 1) + 64))
    try:
        gen = torch.Generator(device="cuda").manual_seed(2)
        token = lambda n: torch.randn(n, model.hidden, generator=gen, device="cuda").bfloat16()  # noqa: E731
        lengths = {i: int(rng.integers(5, 300)) for i in range(a.requests)}
        adapter = {i: int(rng.integers(-1, 4)) for i in lengths}
        model.cache.add(list(lengths))
        for it in range(a.iterations):
            if it == a.iterations // 2:  # request 0 goes on in three ways; every other request ends
                model.cache.fork(0, [1000, 1001, 1002])
                for i in (1000, 1001, 1002):
                    lengths[i], adapter[i] = 1, adapter[0]
                ended = [i for i in lengths if i < 1000 and i % 2]
                model.cache.free(ended)
                for i in ended:
                    del lengths[i], adapter[i]
                moved, used = model.cache.compact(), model.cache.stats()
                model.cache.set_limit(min(used.limit, used.pages_end + len(lengths) * (a.iterations // 64 + 2) + 64))
                print(f"{len(ended)} requests ended, {moved} pages moved, {used.pages_used} in use, {used.pages_shared} of them shared")
            ids = list(lengths)
            lens = [lengths[i] for i in ids]
            x = token(sum(lens))
            torch.cuda.synchronize()
            t = time.perf_counter()
            y = model.step(x, ids, [adapter[i] for i in ids], lens)
            torch.cuda.synchronize()
            print(f"iteration {it}: {len(ids)} requests, {sum(lens)} tokens, {1e3 * (time.perf_counter() - t):.2f} ms, output rms {float(y.float().square().mean().sqrt()):.3f}")
            lengths = {i: 1 for i in ids}
        return model.cache.stats()
    finally:
        model.close()


if __name__ == "__main__":
    main()
