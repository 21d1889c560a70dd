"""Batches whose requests share prefixes (lora_kv_batch_create_shared): attention against its definition in 64 bits, request by request, and what the batch is cut
into.  Forks of prompts, forks of forks, requests that share nothing beside them; all types of pages; one token and several; pages that end inside everything."""
import math

import numpy as np
import pytest

import kv_e4m3_plain
import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _mods():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache
    return B, KvCache


class Tree:
    """Requests given as (parent, tokens of the parent or -1, own cached tokens, new tokens); a request with 0 new tokens is no part of the batch but keeps its pages."""

    def __init__(self, requests, heads, kv, dim, page=64, kind="bf16", seed=0, layers=1, shared=256, beyond=None, order=None, **kw):
        B, KvCache = _mods()
        self.B, self.heads, self.kv, self.dim, self.page, self.kind = B, heads, kv, dim, page, kind
        length = []
        for p, n, own, _new in requests:
            length.append((0 if p is None else length[p] if n < 0 else n) + own)
        need = sum(-(-(r[2] + r[3]) // page) + 2 for r in requests) + 2  # (a fork's first page may be a copy)
        self.cache = KvCache(layers, heads, kv, dim, need, page_tokens=page, max_seqs=len(requests) + 1, max_batch_seqs=len(requests) + 1,
                             max_batch_tokens=max(1, sum(r[3] for r in requests)), dtype=B.LORA_F32 if kind == "f32" else B.LORA_BF16, e4m3=kind == "e4m3", **kw)
        for i, (p, n, own, _new) in enumerate(requests):
            if p is None:
                self.cache.add(i)
            else:
                self.cache.fork(p, i, n)
            self.cache.extend(i, own)
        self.ids = [i for i, r in enumerate(requests) if r[3]]
        if order:
            self.ids = [self.ids[k] for k in np.random.default_rng(order).permutation(len(self.ids))]
        self.ctx, new = [length[i] for i in self.ids], [requests[i][3] for i in self.ids]
        self.offsets = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.batch = self.cache.batch(np.asarray(self.ids), self.offsets, shared=shared)
        self.dt = torch.float32 if kind == "f32" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shape = self.cache.pages.shape
        if kind == "e4m3":
            split = 2 * kv * page * dim
            self.host = torch.empty(shape, dtype=torch.uint8)
            self.host[..., :split] = (torch.randn(*shape[:2], split, generator=gen, device="cuda") * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).cpu()
            self.host[..., split:] = torch.randint(118, 123, self.host[..., split:].shape, generator=gen, dtype=torch.uint8, device="cuda").cpu()
        else:
            self.host = torch.randn(shape, generator=gen, device="cuda").to(self.dt).cpu()
        if beyond is not None:
            kept = torch.full_like(self.host, beyond)
            for i, c, n in zip(self.ids, self.ctx, new):
                table, whole = self.cache.pages_of(i), (c + n) // page
                kept[table[:whole]] = self.host[table[:whole]]
                if (c + n) % page:
                    p, m = int(table[whole]), (c + n) % page
                    assert kind == "bf16"
                    a, b = kept[p].view(layers, 2, kv, -1), self.host[p].view(layers, 2, kv, -1)
                    a[:, 0].view(layers, kv, dim // 8, page, 8)[:, :, :, :m] = b[:, 0].view(layers, kv, dim // 8, page, 8)[:, :, :, :m]
                    for t in range(m):
                        a[:, 1].view(layers, kv, page // 8, dim, 8)[:, :, t // 8, :, t % 8] = b[:, 1].view(layers, kv, page // 8, dim, 8)[:, :, t // 8, :, t % 8]
            self.host = kept
        self.cache.pages.copy_(self.host)
        self.q = torch.randn(int(self.offsets[-1]), heads, dim, generator=gen, device="cuda").to(self.dt).cpu()

    def info(self):
        rc, info = self.B.lora_kv_batch_prefixes(self.batch)
        assert rc == 0
        return info

    def keys_values(self, i, layer, g, n):
        table = self.cache.pages_of(i)
        if self.kind == "e4m3":
            return kv_e4m3_plain.read(self.host.numpy(), table, layer, g, self.kv, self.page, self.dim, n)
        if not hasattr(self, "values"):
            self.values = self.host.float().numpy()
        return kv_plain.read(self.values, table, layer, g, self.page, self.dim, 4 if self.kind == "f32" else 8, n)

    def run(self, layer=0, scale=None, batch=None, q=None, out=None):
        q = self.q.cuda() if q is None else q
        out = torch.full(q.shape, float("nan"), dtype=self.dt, device="cuda") if out is None else out
        self.cache.attend(self.batch if batch is None else batch, layer, q, out, 1.0 / math.sqrt(self.dim) if scale is None else scale)
        return out

    def check(self, layer=0, out=None):
        scale = 1.0 / math.sqrt(self.dim)
        out = self.run(layer) if out is None else out
        torch.cuda.synchronize()
        got, q, eps = out.float().cpu().numpy(), self.q.float().numpy(), 2.0**-24
        for j, i in enumerate(self.ids):
            rows, c, n = slice(int(self.offsets[j]), int(self.offsets[j + 1])), self.ctx[j], int(self.offsets[j + 1] - self.offsets[j])
            for g in range(self.kv):
                k, v = self.keys_values(i, layer, g, c + n)
                for h in range(g * (self.heads // self.kv), (g + 1) * (self.heads // self.kv)):
                    want, mass, reach = kv_plain.attend(q[rows, h], k, v, c, scale)
                    # scores off by dim products' roundings, sums over the tokens by an ulp a step; parts are joined with a weight of a few roundings more.  With bf16 every
                    # weight is off by 2^-8 of itself besides, and the output by half a step
                    f32 = mass * ((2 * self.dim + 8) * eps * reach[..., None] + (c + n + 32) * 2 * eps)
                    bound = f32 if self.kind == "f32" else f32 + 2.0**-8 * mass + 2.0**-8 * (np.abs(want) + 2.0**-7 * mass) + 1e-38
                    over = np.abs(got[rows, h] - want) - bound
                    assert np.isfinite(got[rows, h]).all() and (over <= 0).all(), (i, h, np.unravel_index(np.argmax(over), over.shape), float(over.max()))
        return out

    def close(self):
        self.cache.close()


def _check(requests, heads, kv, dim, prefixes=None, segments=None, **kw):
    layer = kw.pop("layer", 0)
    t = Tree(requests, heads, kv, dim, **kw)
    try:
        info = t.info()
        if prefixes is not None:
            assert info.n_prefixes == prefixes, (info.n_prefixes, info.n_segments)
        if segments is not None:
            assert info.n_segments == segments
        t.check(layer)
    finally:
        t.close()


def forks(n, prefix, own, new=lambda i: 1):
    """n forks of one prompt, own(i) tokens of their own cached; the prompt itself is no part of the batch"""
    return [(None, -1, prefix, 0)] + [(0, -1, own(i), new(i)) for i in range(n)]


KINDS = ["bf16", "f32", "e4m3"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64), (256, 32), (128, 256), (64, 128), (256, 64)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (5, 1)])
def test_forks_of_a_prompt(heads, kv, dim, page, kind):
    _check(forks(3, 700, lambda i: 37 * i), heads, kv, dim, 1, 3, page=page, kind=kind, seed=1)
    _check(forks(20, 512, lambda i: i % 3, lambda i: 1 + i % 2), heads, kv, dim, 1, 20, page=page, kind=kind, seed=2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kv,dim", [(16, 2, 128), (17, 1, 64), (32, 1, 128), (20, 4, 64), (130, 1, 64), (8, 8, 64), (7, 7, 128), (16, 1, 256)])
def test_groups_of_every_kind(heads, kv, dim, kind):
    # (130 heads of one key-value head are a tile of their own: nothing to share)
    most = heads // kv < 128
    _check(forks(7, 900, lambda i: 30 * i), heads, kv, dim, int(most), 7 * most, page=32, kind=kind, seed=3)


@pytest.mark.parametrize("kind", KINDS)
def test_several_tokens_each_and_prompts_beside(kind):
    """Drafts of a few tokens, a continuation long enough for tiles of its own, requests that share nothing, in an order that has nothing to do with who shares what."""
    requests = forks(9, 600, lambda i: 11 * i, lambda i: (1, 2, 5, 31, 1, 9, 40, 1, 3)[i]) + [(None, -1, 300, 1), (None, -1, 0, 200), (None, -1, 5, 1), (0, 600, 0, 300), (0, 320, 1, 1)]
    # 300 tokens of 2 query heads a key-value head are tiles of their own; the last shares 320 tokens of the 600 with the nine, two prefixes then
    _check(requests, 4, 2, 64, kind=kind, seed=4, order=1, segments=10)
    _check(requests, 4, 2, 128, kind=kind, seed=5, order=2, page=32, segments=10)
    _check(requests, 8, 8, 64, kind=kind, seed=6, order=3, segments=10)


@pytest.mark.parametrize("kind", KINDS)
def test_prefixes_branch(kind):
    """A system prompt, prompts behind it, conversations behind those: three levels."""
    requests = [(None, -1, 512, 0), (0, -1, 400, 0), (0, -1, 600, 0)]
    requests += [(1, -1, 5 * i, 1) for i in range(4)] + [(2, -1, 300, 1)] + [(2, -1, 7 * i, 2) for i in range(3)] + [(0, -1, 50, 1), (0, 256, 3, 1), (None, -1, 90, 1)]
    requests += [(7, -1, 4, 1), (7, -1, 70, 1)]  # forks of the fourth request behind 2: 512 + 600 + 300 tokens of it
    _check(requests, 8, 2, 64, kind=kind, seed=7, order=4)
    _check(requests, 8, 2, 128, kind=kind, seed=8, page=32, order=5)


@pytest.mark.parametrize("kind", KINDS)
def test_a_chain_of_forks(kind):
    """Every request is a fork of the one before it with tokens of its own: prefixes of prefixes, more than are told apart."""
    requests = [(None, -1, 64, 1)] + [(i, -1, 96 + 64 * (i % 3), 1) for i in range(40)]
    _check(requests, 4, 1, 64, kind=kind, page=32, seed=9)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("prefix,n,heads,kv,dim", [(9000, 3, 8, 1, 128), (20000, 40, 16, 2, 64), (2500, 90, 8, 2, 64), (4100, 5, 4, 1, 256), (70000, 2, 2, 1, 64)])
def test_long_prefixes_are_cut(prefix, n, heads, kv, dim, kind):
    t = Tree(forks(n, prefix, lambda i: (37 * i) % 250), heads, kv, dim, kind=kind, seed=10)
    try:
        info = t.info()
        assert info.n_prefixes == 1 and info.n_segments == n and info.n_row_items + info.n_tile_items > 1 and info.n_tokens == prefix // 64 * 64
        t.check()
    finally:
        t.close()


def test_large_tiles_of_shared_rows():
    """Rows enough for the tiles of 256 rows: 400 requests with 8 query heads to a key-value head over 12000 tokens, and a prompt long enough beside them."""
    B, _K = _mods()
    for kind in ("bf16", "e4m3"):
        t = Tree(forks(400, 12000, lambda i: i % 40) + [(None, -1, 0, 4096)], 64, 8, 128, kind=kind, seed=11)
        try:
            info = B.lora_kv_batch_info(t.batch)[1]
            assert t.info().n_segments == 400 and (kind != "bf16" or info.tiles_way == B.LORA_KV_TILES_TURNS)
            # a few of the requests, request by request
            t.run()
            out = t.run()
            torch.cuda.synchronize()
            got, q = out.float().cpu().numpy(), t.q.float().numpy()
            for j in (0, 1, 15, 16, 31, 32, 255, 256, 399):
                c = t.ctx[j]
                for h in (0, 7, 8, 63):
                    k, v = t.keys_values(t.ids[j], 0, h // 8, c + 1)
                    want, mass, _r = kv_plain.attend(q[j : j + 1, h], k, v, c, 1 / math.sqrt(128))
                    assert (np.abs(got[j, h] - want[0]) <= (2.0**-7 + 2.0**-10) * mass[0]).all(), (kind, j, h)
            plainly = t.cache.batch(np.asarray([0]), np.asarray([0, 0], np.int32))
            t.cache.batch_destroy(plainly)
        finally:
            t.close()


def test_what_no_request_holds_is_never_used():
    for byte in (float("nan"), float("inf")):
        _check(forks(12, 700, lambda i: 9 * i), 8, 2, 64, kind="bf16", seed=12, beyond=byte)
        _check(forks(40, 300, lambda i: 1), 8, 2, 128, kind="bf16", seed=13, beyond=byte, page=32)


def test_values_that_are_no_numbers():
    """A NaN in a shared token spoils every request that shares it; one in a request's own token that request alone; an infinite value comes out infinite."""
    t = Tree(forks(10, 600, lambda i: 20), 4, 2, 64, seed=14)
    try:
        clean = t.check()
        table = t.cache.pages_of(3)

        def put(page, token, value, half):
            x = t.cache.pages[int(page), 0, half]
            (x.view(2, 8, 64, 8)[0, 0, token, 0] if half == 0 else x.view(2, 8, 64, 8)[0, token // 8, 5, token % 8]).fill_(value)

        put(table[-1], 0, float("nan"), 0)  # request 3's own first token of its last page
        out = t.run()
        j = t.ids.index(3)
        assert torch.isnan(out[j, :2]).all() and torch.isfinite(out[j, 2:]).all()
        others = [k for k in range(10) if k != j]
        assert torch.equal(out[others], clean[others])
        t.cache.pages.copy_(t.host)
        put(table[2], 7, float("inf"), 1)
        out = t.run()
        assert torch.isinf(out[:, :2, 5]).all() and torch.isfinite(out[:, 2:]).all()
        put(table[2], 9, float("nan"), 0)
        out = t.run()
        assert torch.isnan(out[:, :2]).all() and torch.equal(out[:, 2:], clean[:, 2:])
    finally:
        t.close()


def test_values_that_are_no_numbers_in_prefixes_of_few_rows():
    """The same where a wavefront has all rows of a prefix."""
    for kind, bad in (("bf16", float("nan")), ("bf16", float("inf")), ("e4m3", 127)):
        t = Tree(forks(3, 600, lambda i: 20), 4, 2, 64, kind=kind, seed=14)
        try:
            clean = t.check()
            page = int(t.cache.pages_of(2)[3])
            if kind == "e4m3":
                t.cache.pages[page, 0, 2 * 64 * 64 + 7 * 16 + 3] = bad  # head 0's value 7 of token 3
            else:
                t.cache.pages[page, 0, 1].view(2, 8, 64, 8)[0, 0, 7, 3] = bad
            out = t.run()
            assert not torch.isfinite(out[:, :2, 7]).any() and torch.isfinite(out[:, :2, :7]).all() and torch.isfinite(out[:, :2, 8:]).all() and torch.equal(out[:, 2:], clean[:, 2:]), kind
        finally:
            t.close()


def test_outputs_in_place_of_queries_and_strides():
    """Rows of several segments are gathered while others' outputs are written: outputs may take the queries' place, and both may lie in wider rows."""
    for kind in KINDS:
        t = Tree(forks(30, 600, lambda i: i) + [(None, -1, 100, 70), (None, -1, 50, 1)], 4, 2, 64, kind=kind, seed=20, order=1)
        try:
            want = t.run()
            q = t.q.cuda()
            t.run(q=q, out=q)
            assert torch.equal(q, want)
            wide = torch.zeros(len(q), 7, 64, device="cuda", dtype=t.dt)
            wide[:, 1:5] = t.q.cuda()
            out = torch.full((len(q), 6, 64), 3.0, device="cuda", dtype=t.dt)
            t.run(q=wide[:, 1:5], out=out[:, 2:])
            assert torch.equal(out[:, 2:], want) and bool((out[:, :2] == 3).all())
        finally:
            t.close()


def test_rows_whose_scores_leave_nothing():
    """Scores that are all -inf have no softmax, as without prefixes; where one of a row's tokens has a number, it has all the weight."""
    t = Tree(forks(6, 400, lambda i: 10), 2, 1, 64, seed=15)
    try:
        t.cache.pages[:, 0, 0].fill_(float("-inf"))
        q = torch.ones(6, 2, 64, device="cuda").bfloat16()
        out = t.run(q=q)
        assert torch.isnan(out).all()
        # request 2's newest token gets a key of zeros
        table = t.cache.pages_of(3)
        at = (t.ctx[2]) % 64
        t.cache.pages[int(table[-1]), 0, 0].view(1, 8, 64, 8)[0, :, at] = 0
        out = t.run(q=q)
        want = t.host[int(table[-1]), 0, 1].view(1, 8, 64, 8)[0, at // 8, :, at % 8]
        assert torch.equal(out[2].cpu(), want.expand(2, 64)) and torch.isnan(out[[0, 1, 3, 4, 5]]).all()
    finally:
        t.close()


@pytest.mark.parametrize("kind", KINDS)
def test_batches_in_a_row_and_layers(kind):
    """Iterations of appends and attention on shared batches give what batches that share nothing give, to rounding; the same call gives the same bits."""
    B, KvCache = _mods()
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    caches = [KvCache(2, 8, 2, 64, 200, page_tokens=32, max_seqs=40, max_batch_seqs=40, max_batch_tokens=1000, dtype=B.LORA_F32 if kind == "f32" else B.LORA_BF16, e4m3=kind == "e4m3")
              for _ in range(2)]
    try:
        gen = torch.Generator(device="cuda").manual_seed(1)
        rope = torch.randn(900, 64, generator=gen, device="cuda").clamp(-1, 1)
        w = torch.rand(64, generator=gen, device="cuda") + 0.5
        for c in caches:
            c.add(0)
        lengths = {0: 700}
        rng = np.random.default_rng(3)
        for it in range(6):
            if it == 1:
                for c in caches:
                    c.fork(0, np.arange(1, 20))
                lengths = {i: 1 for i in range(20)}
            if it == 4:
                for c in caches:
                    c.free(np.arange(0, 20, 2))
                    c.fork(1, np.arange(30, 35), 690)
                    c.compact()
                lengths = {i: 1 for i in list(range(1, 20, 2)) + list(range(30, 35))}
            ids = np.asarray([int(i) for i in rng.permutation(list(lengths))])
            off = np.concatenate([[0], np.cumsum([lengths[i] for i in ids])]).astype(np.int32)
            T = int(off[-1])
            plans = [c.batch(ids, off, shared=256 if k == 0 else False) for k, c in enumerate(caches)]
            assert (B.lora_kv_batch_prefixes(plans[0])[1].n_prefixes > 0) == (it > 0) and B.lora_kv_batch_prefixes(plans[1])[1].n_prefixes == 0
            for layer in range(2):
                x = torch.randn(T, 12, 64, generator=gen, device="cuda").to(dt)
                outs = []
                for c, plan in zip(caches, plans):
                    q, out = torch.empty(T, 8, 64, device="cuda", dtype=dt), torch.empty(2, T, 8, 64, device="cuda", dtype=dt)
                    c.append(plan, layer, x[:, 8:10], x[:, 10:], q=x[:, :8], q_out=q, rope=rope, q_norm=w, k_norm=w)
                    c.attend(plan, layer, q, out[0], 0.125)
                    c.attend(plan, layer, q, out[1], 0.125)
                    assert torch.equal(out[0], out[1])
                    outs.append(out[0].float())
                err = (outs[0] - outs[1]).norm() / outs[1].norm()
                # each is off by 2^-9 in the root mean square of its roundings at most, twice; fp32 by a few hundred roundings
                assert float(err) <= (1e-5 if kind == "f32" else 2.0**-7), (it, layer, float(err))
            for c, plan in zip(caches, plans):
                c.batch_destroy(plan)
            lengths = {int(i): int(rng.integers(1, 4)) for i in ids}
    finally:
        for c in caches:
            c.close()


def test_captured_and_replayed():
    t = Tree(forks(20, 900, lambda i: 31 * i), 8, 2, 128, seed=16)
    try:
        q, out = t.q.cuda(), torch.empty_like(t.q, device="cuda")
        t.run(q=q, out=out)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            t.cache.attend(t.batch, 0, q, out, 0.1, stream=side)
        for i in range(3):
            q.copy_(torch.randn(q.shape, device="cuda"))
            want = torch.empty_like(out)
            t.cache.attend(t.batch, 0, q, want, 0.1)
            torch.cuda.synchronize()
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), i
    finally:
        t.close()


def test_what_is_shared():
    """What counts as a prefix: pages that are full, of two segments at least, in the batch, of few rows, and enough of them."""
    B, _K = _mods()

    def info(requests, heads=4, kv=2, **kw):
        t = Tree(requests, heads, kv, 64, **kw)
        try:
            i = t.info()
            return i.n_prefixes, i.n_segments, i.n_tokens
        finally:
            t.close()

    assert info(forks(2, 640, lambda i: 1)) == (1, 2, 640)
    assert info(forks(2, 640 + 63, lambda i: 0)) == (1, 2, 640)      # the last page is copied as they write
    assert info(forks(1, 640, lambda i: 1)) == (0, 0, 0)              # its holder is no part of the batch
    assert info(forks(2, 64, lambda i: 600)) == (0, 0, 0)             # too short
    assert info(forks(2, 640, lambda i: 1, lambda i: 64)) == (0, 0, 0)  # tiles of their own
    assert info(forks(2, 640, lambda i: 1, lambda i: 63)) == (1, 2, 640)
    assert info(forks(5, 640, lambda i: 1), shared=False) == (0, 0, 0)
    assert info(forks(2, 352, lambda i: 5), page=32) == (1, 2, 320)   # 11 pages of 32: pieces begin at multiples of 64
    assert info([(None, -1, 640, 1), (0, -1, 0, 1)]) == (1, 2, 640)   # a parent in the batch
    assert info([(None, -1, 700, 1), (None, -1, 700, 1)]) == (0, 0, 0)
    assert info([(None, -1, 320, 0), (0, -1, 320, 0)] + [(1, -1, i, 1) for i in range(3)] + [(0, -1, i, 1) for i in range(3)]) == (2, 6, 640)


def test_what_is_worth_it():
    """Without a number of tokens the library shares what saves more bytes than the parts cost: 2 or 64 requests, long prefixes and short ones."""
    def prefixes(n, tokens, heads, kv, shared, **kw):
        t = Tree(forks(n, tokens, lambda i: 3), heads, kv, 128, shared=shared, **kw)
        try:
            return t.info().n_prefixes
        finally:
            t.close()

    for kind, times in (("bf16", 1), ("e4m3", 2)):
        assert prefixes(64, 704 * times, 32, 8, True, kind=kind) == 1 and prefixes(64, 512 * times, 32, 8, True, kind=kind) == 0
        assert prefixes(2, 1024 * times, 40, 40, True, kind=kind) == 1 and prefixes(2, 512 * times, 40, 40, True, kind=kind) == 0
        assert prefixes(2, 64, 40, 40, 64, kind=kind) == 1 and prefixes(2, 64, 40, 40, 65, kind=kind) == 0 and prefixes(2, 64, 40, 40, 1, kind=kind) == 1
    _check(forks(64, 1024, lambda i: i % 50), 32, 8, 128, 1, 64, kind="bf16", shared=True, seed=18)
    _check(forks(3, 130, lambda i: i), 4, 2, 64, 1, 3, kind="bf16", shared=1, seed=19)


def test_no_room_for_the_parts():
    """More rows than the memory for partial results has room for: the requests are worked on one by one, as if nothing were shared."""
    t = Tree(forks(520, 300, lambda i: 1), 64, 64, 256, page=32, seed=17)
    try:
        assert t.info().n_prefixes == 0
        out = t.run()
        torch.cuda.synchronize()
        for j in (0, 519):
            k, v = t.keys_values(t.ids[j], 0, 5, t.ctx[j] + 1)
            want, mass, _r = kv_plain.attend(t.q[j : j + 1, 5].float().numpy(), k, v, t.ctx[j], 1 / 16)
            assert (np.abs(out[j, 5].float().cpu().numpy() - want[0]) <= (2.0**-7 + 2.0**-10) * mass[0]).all()
    finally:
        t.close()


def test_refusals():
    B, KvCache = _mods()
    cache = KvCache(1, 2, 2, 64, 8, page_tokens=32, max_seqs=3, max_batch_seqs=2, max_batch_tokens=40)
    try:
        cache.add([0, 1, 2])
        create = B.lora_kv_batch_create_shared
        assert create(cache.handle, [0, 0], [0, 1, 2])[0] == B.LORA_E_INVAL and create(cache.handle, [7], [0, 1])[0] == B.LORA_E_NOTFOUND
        assert create(cache.handle, [0, 1], [0, 2, 1])[0] == B.LORA_E_INVAL and create(cache.handle, [0, 1, 2], [0, 1, 2, 3])[0] == B.LORA_E_NOMEM
        assert create(cache.handle, [0], [0, 41])[0] == B.LORA_E_NOMEM and create(None, [0], [0, 1])[0] == B.LORA_E_INVAL
        assert create(cache.handle, [0], [0, 1], -1)[0] == B.LORA_E_INVAL
        b = cache.batch([0], [0, 0], shared=True)
        assert B.lora_kv_batch_prefixes(b)[1].n_prefixes == 0
        cache.batch_destroy(b)
        assert B.lora_kv_batch_prefixes(b)[0] == B.LORA_E_INVAL and B.lora_kv_batch_prefixes(None)[0] == B.LORA_E_INVAL
    finally:
        cache.close()


def test_numbers_of_tokens_beyond_32_bits():
    """They are none, or negative: not what is left of them."""
    B, _K = _mods()
    t = Tree(forks(2, 640, lambda i: 1), 4, 2, 64, shared=2**32 + 1)
    try:
        assert t.info().n_prefixes == 0
        for n in (-1, -(2**32) + 1):
            with pytest.raises(B.LoraError):
                t.cache.batch([1], [0, 1], shared=n)
    finally:
        t.close()
