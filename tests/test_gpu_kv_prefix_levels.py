"""Prefixes of prefixes: how many levels a batch has, what is left out where there is no room, and attention over all of them request by request."""
import math

import numpy as np
import pytest

import kv_plain
import test_gpu_kv_prefixes as prefixes

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

KINDS = prefixes.KINDS


def _tree(requests, heads, kv, dim, max_batch_tokens, **kw):
    """prefixes.Tree in a cache of that many batch tokens"""
    mods = prefixes._mods
    B, KvCache = mods()
    prefixes._mods = lambda: (B, lambda *a, **k: KvCache(*a, **{**k, "max_batch_tokens": max_batch_tokens}))
    try:
        return prefixes.Tree(requests, heads, kv, dim, **kw)
    finally:
        prefixes._mods = mods


def _check(t):
    """Attention by its definition.  Of bf16 weights, segments with up to 16 rows have 16 bits: off by 2^-16; the others by 2^-8."""
    out, group = t.run(), t.heads // t.kv
    torch.cuda.synchronize()
    got, q, eps = out.float().cpu().numpy(), t.q.float().numpy(), 2.0**-24
    for j, i in enumerate(t.ids):
        rows, c, n = slice(int(t.offsets[j]), int(t.offsets[j + 1])), t.ctx[j], int(t.offsets[j + 1] - t.offsets[j])
        for g in range(t.kv):
            k, v = t.keys_values(i, 0, g, c + n)
            for h in range(g * group, (g + 1) * group):
                want, mass, reach = kv_plain.attend(q[rows, h], k, v, c, 1.0 / math.sqrt(t.dim))
                # scores off by dim products' roundings, sums over the tokens by two roundings a step, joins by a few more
                bound = mass * ((2 * t.dim + 8) * eps * reach[..., None] + (c + n + 32) * 2 * eps)
                if t.kind != "f32":
                    bound = bound + (2.0**-16 if n * group <= 16 else 2.0**-8) * mass
                    bound = bound + 2.0**-8 * (np.abs(want) + bound) + 1e-38
                over = np.abs(got[rows, h] - want) - bound
                assert (over <= 0).all(), (i, h, np.unravel_index(np.argmax(over), over.shape), float(over.max()))


def _levels(requests, heads, kv, dim, max_batch_tokens, want, **kw):
    """want: prefixes, segments that have one, tokens of all prefixes"""
    t = _tree(requests, heads, kv, dim, max_batch_tokens, **kw)
    try:
        info = t.info()
        assert (info.n_prefixes, info.n_segments, info.n_tokens) == want
        _check(t)
    finally:
        t.close()


# Ten requests, each a fork of the one before it with 256 tokens more: all share 256 tokens, nine the next 256, ..., two the ninth
CHAIN = [(None, -1, 256, 1)] + [(i, -1, 256, 1) for i in range(9)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 64, 64), (4, 4, 128, 32), (8, 1, 256, 128), (16, 1, 64, 256)])
def test_seven_levels_and_no_more(heads, kv, dim, page, kind):
    _levels(CHAIN, heads, kv, dim, 100, (7, 10, 7 * 256), page=page, kind=kind, seed=31, order=1)


@pytest.mark.parametrize("kind", KINDS)
def test_prefixes_without_room_are_left_out_and_those_behind_them_are_not(kind):
    """The prefixes' segments may have 2 * max_batch_tokens tokens in all."""
    # room for 20: the 10 of the first and the 9 of the second, 1 left
    _levels(CHAIN, 8, 2, 64, 10, (2, 10, 512), kind=kind, seed=32)
    # room for 24: 5 left, which 8, 7 and 6 do not fit into; the 5 that share 1536 tokens do, from the 512 on that they have already
    _levels(CHAIN, 8, 2, 64, 12, (3, 10, 1536), kind=kind, seed=33)
    # room for 22: 3 left, for the 3 that share 2048
    _levels(CHAIN, 8, 2, 128, 11, (3, 10, 2048), kind=kind, seed=34, page=32)


@pytest.mark.parametrize("n,want", [(21, (3, 21, 19 * 64)), (22, (2, 22, 2 * 64))])
def test_what_is_behind_many_prefixes_without_room(n, want):
    """n requests, each a fork of the one before it with 64 tokens more, room for 2 n + 2: n share the first 64 tokens, n - 1 the next, 3 places are left.  Three requests are n - 5 prefixes on: found
    behind 16, not behind 17."""
    _levels([(None, -1, 64, 1)] + [(i, -1, 64, 1) for i in range(n - 1)], 4, 4, 64, n + 1, want, shared=64, seed=39)


@pytest.mark.parametrize("kind", KINDS)
def test_three_levels_that_branch(kind):
    """A system prompt, two prompts behind it, conversations behind those; one that forks early, one that shares nothing."""
    requests = [(None, -1, 512, 0), (0, -1, 512, 0), (0, -1, 768, 0)]
    requests += [(1, -1, 5 * i, 1) for i in range(4)] + [(2, -1, 300, 1)] + [(2, -1, 7 * i, 2) for i in range(3)] + [(0, -1, 50, 1), (0, 256, 3, 1), (None, -1, 90, 1)]
    requests += [(7, -1, 4, 1), (7, -1, 70, 1)]  # of the request behind 2 with 300 tokens of its own, 256 of which are theirs too
    # 256 tokens that 12 segments share; 256 more that 11 do; 512 behind those of 4, 768 of 6, and 256 behind these of 3
    for heads, kv, dim, page in ((8, 2, 64, 64), (4, 4, 128, 32), (16, 1, 64, 64)):
        _levels(requests, heads, kv, dim, 100, (5, 12, 256 + 256 + 512 + 768 + 256), page=page, kind=kind, seed=35, order=4)


def test_tiles_three_to_a_compute_unit_with_prefixes():
    """Segments of more than 16 rows, tiles enough for three blocks on a compute unit: shared rows go there too."""
    B, _K = prefixes._mods()
    t = _tree(prefixes.forks(120, 512, lambda i: 3 * (i % 7), lambda i: 5 + i % 3), 32, 8, 128, 2000, seed=36, order=2)
    try:
        info = B.lora_kv_batch_info(t.batch)[1]
        assert info.tiles_way == B.LORA_KV_TILES_MANY and t.info().n_tile_items and t.info().n_segments == 120
        _check(t)
    finally:
        t.close()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_tiles_of_256_rows_with_prefixes(kind):
    """Shared rows enough for the tiles of 256 rows over pages of both types: of one token each, and of more rows than a row item has."""
    B, _K = prefixes._mods()
    for new in (1, 5):
        t = _tree(prefixes.forks(64, 40000, lambda i: i % 40, lambda i: new), 32, 8, 128, 2000, kind=kind, seed=37)
        try:
            assert B.lora_kv_batch_info(t.batch)[1].tiles_way == B.LORA_KV_TILES_TURNS and t.info().n_segments == 64
            out = t.run()
            got, q = out.float().cpu().numpy(), t.q.float().numpy()
            for j in (0, 1, 31, 32, 63):  # a few of the requests
                c, rows = t.ctx[j], slice(int(t.offsets[j]), int(t.offsets[j + 1]))
                for h in (0, 7, 30):
                    k, v = t.keys_values(t.ids[j], 0, h // 4, c + new)
                    want, mass, reach = kv_plain.attend(q[rows, h], k, v, c, 1 / math.sqrt(128))
                    bound = mass * (264 * 2.0**-24 * reach[..., None] + (c + new + 32) * 2.0**-23 + (2.0**-16 if new == 1 else 2.0**-8))
                    bound = bound + 2.0**-8 * (np.abs(want) + bound)
                    assert (np.abs(got[rows, h] - want) <= bound).all(), (new, j, h)
        finally:
            t.close()


def test_shared_batches_on_two_streams():
    """Batches and calls on streams in turn, with nothing between them but the cache's own order."""
    t = _tree(prefixes.forks(20, 700, lambda i: 5 * i), 8, 2, 64, 100, seed=38)
    try:
        want = t.run()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        q = t.q.cuda()
        torch.cuda.synchronize()
        outs = []
        for i in range(6):
            t.cache.truncate(t.ids, t.ctx)
            batch = t.cache.batch(np.asarray(t.ids), t.offsets, shared=256, stream=streams[i % 2])
            with torch.cuda.stream(streams[(i + 1) % 2]):
                out = torch.full_like(q, float("nan"))
                t.cache.attend(batch, 0, q, out, 1.0 / 8)
            outs.append(out)
            t.cache.batch_destroy(batch)
        torch.cuda.synchronize()
        assert all(torch.equal(out, want) for out in outs)
    finally:
        t.close()
