"""lora_kv_attend against its definition in 64 bits: requests of one token and prompts, grouped heads, page sizes, head sizes, both types, lengths
around every boundary (chunks, products, tiles, pages, pieces), strides, whatever lies beyond a token's position."""
import math

import numpy as np
import pytest

import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _mods():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache
    return B, KvCache


class Setup:
    """Sequences with scattered pages and a batch: segs is [(cached tokens, new tokens)]."""

    def __init__(self, segs, heads, kv, dim, page=64, dtype="bf16", seed=0, layers=1, fill=1.0, beyond=None):
        B, KvCache = _mods()
        self.segs, self.heads, self.kv, self.dim, self.page, self.layers = segs, heads, kv, dim, page, layers
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.u = 8 if dtype == "bf16" else 4
        need = [-(-(c + n) // page) for c, n in segs]
        n_pages = sum(need) + 3
        self.cache = KvCache(layers, heads, kv, dim, n_pages, page_tokens=page, max_seqs=len(segs) + 1, max_batch_seqs=len(segs) + 1,
                             max_batch_tokens=max(1, sum(n for _c, n in segs)), dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
        ids = np.arange(len(segs))
        self.cache.add(ids)
        ctx = np.asarray([c for c, _n in segs])
        for at in range(0, int(ctx.max()), page):  # page by page in turn: the pages of a sequence lie apart
            who = np.flatnonzero(ctx > at)
            self.cache.extend(who, np.minimum(page, ctx[who] - at))
        self.offsets = np.concatenate([[0], np.cumsum([n for _c, n in segs])]).astype(np.int32)
        self.batch = self.cache.batch(ids, self.offsets)
        self.tables = [self.cache.pages_of(int(i)) for i in ids]
        gen = torch.Generator().manual_seed(seed)
        host = torch.randn(self.cache.pages.shape, generator=gen) * fill
        self.T = sum(n for _c, n in segs)
        self.q = torch.randn(self.T, heads, dim, generator=gen).to(self.dt)
        self.host = host.to(self.dt)
        if beyond is not None:  # everything that no sequence holds
            kept = torch.full(host.shape, float(beyond)).to(self.dt)
            a, b = kept.float().numpy(), self.host.float().numpy()
            for i, (c, n) in enumerate(segs):
                for layer in range(layers):
                    for h in range(kv):
                        if c + n:
                            k, v = kv_plain.read(b, self.tables[i], layer, h, page, dim, self.u, c + n)
                            kv_plain.write(a, self.tables[i], layer, h, page, dim, self.u, 0, k, v)
            self.host = torch.from_numpy(a).to(self.dt)
        self.cache.pages.copy_(self.host)

    def want(self, scale, layer=0, q=None):
        pages, q = self.host.float().numpy(), (self.q if q is None else q).float().numpy()
        out, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
        for i, (c, n) in enumerate(self.segs):
            rows = slice(int(self.offsets[i]), int(self.offsets[i + 1]))
            for h in range(self.heads if n else 0):
                k, v = kv_plain.read(pages, self.tables[i], layer, h // (self.heads // self.kv), self.page, self.dim, self.u, c + n)
                out[rows, h], mass[rows, h], reach[rows, h] = kv_plain.attend(q[rows, h], k, v, c, scale)
        return out, mass, reach

    def bound(self, out, mass, reach):
        """What rounding can do.  fp32: a score of dim products is off by up to dim * 2^-24 of sum |q||k| (twice: scores and their maximum), the
        exponential by an ulp and its argument's rounding, each of the sums over the tokens by an ulp a step.  bf16 besides: every weight is
        rounded to 8 significant bits (a relative error of up to 2^-8) and so is the output."""
        eps = 2.0**-24
        longest = max(c + n for c, n in self.segs)
        f32 = mass * ((2 * self.dim + 8) * eps * reach[..., None] + (longest + 16) * 2 * eps)
        return f32 if self.dt == torch.float32 else f32 + 2.0**-8 * mass + 2.0**-8 * (np.abs(out) + 2.0**-7 * mass) + 1e-38

    def run(self, scale, q=None, layer=0):
        q = (self.q if q is None else q).cuda()
        out = torch.full(q.shape, float("nan"), dtype=self.dt, device="cuda")
        self.cache.attend(self.batch, layer, q, out, scale)
        torch.cuda.synchronize()
        return out

    def check(self, scale=None, layer=0):
        scale = 1.0 / math.sqrt(self.dim) if scale is None else scale
        got = self.run(scale, layer=layer).float().cpu().numpy()
        out, mass, reach = self.want(scale, layer)
        over = np.abs(got - out) - self.bound(out, mass, reach)
        assert np.isfinite(got).all() and (over <= 0).all(), (self.segs, np.unravel_index(np.argmax(over), over.shape), float(over.max()))

    def close(self):
        self.cache.close()


def _check(segs, heads, kv, dim, **kw):
    scale, layer = kw.pop("scale", None), kw.pop("layer", 0)
    s = Setup(segs, heads, kv, dim, **kw)
    try:
        s.check(scale, layer)
    finally:
        s.close()


TOKENS = [(0, 1), (1, 1), (30, 1), (31, 1), (32, 1), (63, 1), (64, 1), (127, 1), (130, 1), (255, 1), (256, 1), (700, 1)]
PROMPTS = [(0, 1), (0, 3), (0, 33), (5, 29), (31, 32), (64, 64), (0, 127), (1, 128), (127, 130), (300, 17), (0, 0), (90, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64), (256, 32), (128, 256), (64, 128), (256, 64)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (5, 1)])
def test_tokens_and_prompts(heads, kv, dim, page, dtype):
    _check(TOKENS, heads, kv, dim, page=page, dtype=dtype, seed=1)
    _check(PROMPTS, heads, kv, dim, page=page, dtype=dtype, seed=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim", [(16, 2, 128), (17, 1, 64), (32, 1, 128), (20, 4, 64), (130, 1, 64), (8, 8, 64), (7, 7, 128)])
def test_groups_of_every_kind(heads, kv, dim, dtype):
    _check([(45, 1), (0, 1), (63, 2), (99, 3), (0, 9), (10, 16), (200, 1)], heads, kv, dim, page=32, dtype=dtype, seed=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("segs,heads,kv,dim", [
    ([(9001, 1)], 8, 1, 128), ([(4999, 1), (0, 1), (3333, 1)], 4, 2, 64), ([(6000, 5)], 2, 2, 128), ([(5000, 40)], 8, 2, 64),
    ([(3000, 200), (12, 1), (2500, 1)], 4, 1, 128), ([(4100, 33)], 2, 1, 256), ([(2047, 1), (2048, 1), (2049, 1)], 40, 8, 64)])
def test_long_caches_are_cut_and_joined(segs, heads, kv, dim, dtype):
    s = Setup(segs, heads, kv, dim, page=64, dtype=dtype, seed=4)
    try:
        B, _K = _mods()
        assert B.lora_kv_batch_info(s.batch)[1].n_joins > 0
        s.check()
    finally:
        s.close()


def test_a_cache_of_many_pages_and_a_long_sequence():
    _check([(131073, 1), (70000, 3)], 2, 1, 64, seed=15)
    _check([(66000, 40)], 2, 2, 64, page=32, seed=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_beyond_4_gb(dtype):
    """Pages whose place in the buffer passes 32 bits, in bytes and in values: read, written, copied and moved."""
    B, KvCache = _mods()
    dt, u = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    kv, dim, page, layers, e = 8, 128, 256, 2, 2 if dtype == "bf16" else 4
    page_bytes = layers * 2 * kv * page * dim * e
    low = (9 << 30) // page_bytes  # 9 GB of pages that another sequence holds
    cache = KvCache(layers, 8, kv, dim, low + 12, page_tokens=page, max_seqs=4, max_batch_seqs=3, max_batch_tokens=1400, dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
    try:
        cache.add([0, 1, 2])
        cache.extend([0], [low * page])
        gen = torch.Generator().manual_seed(1)
        off = np.asarray([0, 900, 1200], np.int32)
        batch = cache.batch([1, 2], off)
        assert min(cache.pages_of(1)) >= low and low * page_bytes > 2**33
        qkv = torch.randn(1200, 24, dim, generator=gen).to(dt)
        dev = qkv.cuda()
        cache.append(batch, 1, dev[:, 8:16], dev[:, 16:])
        out = torch.empty(1200, 8, dim, dtype=dt, device="cuda")

        def look(rows, at, tokens, seqs):
            """Output rows `rows` of `tokens` positions from `at` of the sequences against the definition."""
            got = out.float().cpu().numpy()
            f = qkv.float().numpy()
            for i, r in zip(seqs, rows):
                base = {1: 0, 2: 900, 3: 0}[i]
                for h in (0, 7):
                    want, mass, reach = kv_plain.attend(f[base + at : base + at + tokens, h], f[base : base + at + tokens, 8 + h], f[base : base + at + tokens, 16 + h], at, 0.09)
                    bound = Setup.bound(fake, want, mass, reach)
                    assert (np.abs(got[r : r + tokens, h] - want) <= bound).all(), (i, h)

        fake = type("Shape", (), dict(dt=dt, dim=dim, segs=[(900, 0)]))
        cache.attend(batch, 1, dev[:, :8], out, 0.09)
        torch.cuda.synchronize()
        look([0], 0, 900, [1])
        look([900], 0, 300, [2])
        # one token each, of a fork as well: its last page is copied up there; then everything moves down
        cache.batch_destroy(batch)
        cache.fork(1, [3], 899)
        cache.truncate([1, 2], [899, 299])
        for moved in (False, True):
            if moved:
                cache.truncate([1, 2, 3], [899, 299, 899])
                cache.free([0])
                assert cache.compact() > 0 and max(cache.pages_of(3).max(), cache.pages_of(2).max()) < 12
            one = cache.batch([1, 2, 3], [0, 1, 2, 3])
            k = torch.stack([dev[899], dev[1199], dev[899]])
            cache.append(one, 1, k[:, 8:16], k[:, 16:])
            out.fill_(float("nan"))
            cache.attend(one, 1, k[:, :8], out[:3], 0.09)
            torch.cuda.synchronize()
            look([0], 899, 1, [1])
            look([1], 299, 1, [2])
            look([2], 899, 1, [3])
            cache.batch_destroy(one)
        assert cache.stats().pages_copied > 0
    finally:
        cache.close()


def test_long_prompts():
    _check([(0, 1500), (0, 700)], 4, 2, 128, seed=5)
    _check([(513, 1023)], 3, 3, 64, page=32, seed=6)
    _check([(0, 600)], 2, 1, 128, dtype="f32", seed=6)


# Steps of 32 tokens, by one wavefront or two in turn: every number of them from one to nine, whole and broken, with tokens in the cache and without
STEPS = [(0, 31), (0, 32), (1, 32), (5, 60), (0, 64), (32, 64), (0, 97), (64, 64), (100, 33), (0, 160), (97, 95), (193, 31), (200, 57), (255, 33)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,page", [(2, 2, 64, 32), (6, 2, 64, 128), (2, 1, 128, 32), (4, 4, 128, 256), (4, 1, 256, 32), (2, 2, 256, 64)])
def test_prompts_of_every_number_of_steps(heads, kv, dim, page, dtype):
    for part in (STEPS[:5], STEPS[5:10], STEPS[10:]):
        _check(part, heads, kv, dim, page=page, dtype=dtype, seed=11, beyond=float("nan"))


# Batches for each way of working on tiles: heads of 64 with few tiles, alone and beside single tokens, with a longer tile, with more tiles than compute units; heads of 128
# with two blocks on a compute unit, with three (many tiles, and short ones), single tokens beside both
@pytest.mark.parametrize("segs,heads,kv,dim", [
    ([(0, 1000)], 4, 4, 64), ([(3, 700), (12, 1), (900, 1), (0, 2)], 8, 4, 64), ([(0, 1100)], 4, 4, 64), ([(0, 300), (70, 230), (0, 140)], 40, 40, 64),
    ([(0, 900)], 40, 40, 128), ([(0, 129), (5, 130), (0, 200), (64, 150), (0, 100), (0, 1), (33, 250)], 48, 48, 128), ([(0, 40)] * 26, 32, 32, 128),
    ([(500, 1)] * 9 + [(0, 310)], 64, 8, 128), ([(0, 400), (400, 300)], 32, 32, 256)])
def test_tiles_few_and_many(segs, heads, kv, dim):
    _check(segs, heads, kv, dim, seed=12)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [128, 256])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_prompts_that_grow_along_the_cache(sign, dim, dtype):
    """As below, for the other head sizes: the maximum moves beside products that are under way."""
    s = Setup([(0, 333), (50, 130)], 4, 2, dim, dtype=dtype, seed=13)
    try:
        a = s.host.float().numpy()
        for i, (c, n) in enumerate(s.segs):
            for h in range(s.kv):
                k, v = kv_plain.read(a, s.tables[i], 0, h, s.page, s.dim, s.u, c + n)
                k = np.abs(k) * np.linspace(0.01, 4, c + n)[:, None]
                kv_plain.write(a, s.tables[i], 0, h, s.page, s.dim, s.u, 0, k, v)
        s.host = torch.from_numpy(a).to(s.dt)
        s.cache.pages.copy_(s.host)
        s.q = (s.q.float().abs() * sign).to(s.dt)
        s.check()
    finally:
        s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill,scale", [(30.0, 1.0), (1.0, 1e-6), (8.0, 0.5), (1e-20, 1.0)])
def test_scores_of_every_size(fill, scale, dtype):
    """Weights that are all on one token, all alike, and maxima that keep growing."""
    _check([(500, 1), (0, 300), (77, 40)], 4, 2, 64, dtype=dtype, seed=7, fill=fill, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_that_grow_along_the_cache(sign, dtype):
    """Keys that grow steadily: the running maximum moves in every step, or never after the first."""
    s = Setup([(600, 1), (0, 333), (50, 10)], 4, 2, 64, dtype=dtype, seed=8)
    try:
        a = s.host.float().numpy()
        for i, (c, n) in enumerate(s.segs):
            for h in range(s.kv):
                k, v = kv_plain.read(a, s.tables[i], 0, h, s.page, s.dim, s.u, c + n)
                k = np.abs(k) * np.linspace(0.01, 4, c + n)[:, None]
                kv_plain.write(a, s.tables[i], 0, h, s.page, s.dim, s.u, 0, k, v)
        s.host = torch.from_numpy(a).to(s.dt)
        s.cache.pages.copy_(s.host)
        s.q = (s.q.float().abs() * sign).to(s.dt)
        s.check()
    finally:
        s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("beyond", [float("nan"), float("inf"), -float("inf"), 3e38])
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 128), (256, 64)])
def test_what_no_sequence_holds_has_no_influence(dim, page, beyond, dtype):
    """Pages of nobody, and the rest of each sequence's last page."""
    _check([(0, 1), (33, 1), (0, 5), (70, 1), (10, 50), (0, 130), (600, 1), (250, 9)], 4, 2, dim, page=page, dtype=dtype, seed=9, beyond=beyond)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("segs,at,heads", [([(0, 70)], 41, 4), ([(20, 3)], 21, 2), ([(30, 200)], 150, 8), ([(2500, 60)], 2531, 4), ([(2500, 4)], 2502, 2)])
def test_tokens_behind_a_token_have_no_influence(segs, at, heads, bad, dtype):
    """A key and a value that are no numbers: rows before that token do not see them; rows from it on do."""
    s = Setup(segs, heads, 2, 64, dtype=dtype, seed=10)
    try:
        a = s.host.float().numpy()
        (c, n), scale = s.segs[0], 0.125
        out, mass, reach = s.want(scale)
        k, v = kv_plain.read(a, s.tables[0], 0, 1, s.page, s.dim, s.u, c + n)
        k[at], v[at] = bad, bad
        kv_plain.write(a, s.tables[0], 0, 1, s.page, s.dim, s.u, 0, k, v)
        s.cache.pages.copy_(torch.from_numpy(a).to(s.dt))
        got = s.run(scale).float().cpu().numpy()
        seen, g = at - c, heads // 2
        clean = np.ones(got.shape, bool)
        clean[seen:, g:] = False
        assert np.isfinite(got[clean]).all() and (np.abs(got - out) <= s.bound(out, mass, reach))[clean].all()
        # a NaN key makes a row's weights NaN; an infinite one does where its score is +inf (where it is -inf it has no weight, and its value then
        # gives 0 * inf)
        assert not np.isfinite(got[seen:, g:]).any()
    finally:
        s.close()


def test_layers_and_strides_and_in_place():
    """Queries out of a [T][heads + 2 kv][dim] buffer, outputs into a wider one, and outputs over the queries."""
    s = Setup([(100, 1), (0, 70), (900, 1), (40, 6)], 8, 2, 128, seed=11, layers=3)
    try:
        scale = 0.09
        for layer in range(3):
            out, mass, reach = s.want(scale, layer)
            wide = torch.randn(s.T, 12, 128, device="cuda").bfloat16()
            wide[:, 1:9] = s.q.cuda()
            to = torch.full((s.T, 11, 128), 7.0, dtype=torch.bfloat16, device="cuda")
            s.cache.attend(s.batch, layer, wide[:, 1:9], to[:, 2:10], scale)
            got = to.float().cpu().numpy()
            assert (np.abs(got[:, 2:10] - out) <= s.bound(out, mass, reach)).all()
            assert (got[:, :2] == 7).all() and (got[:, 10:] == 7).all()
            s.cache.attend(s.batch, layer, wide[:, 1:9], wide[:, 1:9], scale)
            assert torch.equal(wide[:, 1:9], to[:, 2:10])
    finally:
        s.close()


def test_the_same_call_gives_the_same_bits():
    s = Setup([(5000, 1), (0, 300), (2000, 30), (77, 1)], 8, 2, 128, seed=12)
    try:
        first = s.run(0.1)
        for _ in range(3):
            assert torch.equal(s.run(0.1), first)
    finally:
        s.close()


def test_streams_follow_each_other():
    """Calls of one cache on two streams: each waits for the one before, and queries written on a call's own stream are seen."""
    s = Setup([(3000, 1), (0, 200)], 8, 2, 128, seed=13)
    try:
        q = s.q.cuda()
        want = s.run(0.1)
        other, out, mid = torch.cuda.Stream(), torch.empty_like(q), torch.empty_like(q)
        torch.cuda.synchronize()
        for _ in range(5):
            out.zero_()
            s.cache.attend(s.batch, 0, q, mid, 0.1)                 # on the current stream
            s.cache.attend(s.batch, 0, q, out, 0.1, stream=other)   # shares the memory for partial results
            s.cache.attend(s.batch, 0, q, mid, 0.1)
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(mid, want)
    finally:
        s.close()


def test_captured_calls_replay():
    s = Setup([(3000, 1), (0, 200), (10, 1)], 8, 2, 128, seed=14)
    try:
        q, out = s.q.cuda(), torch.zeros(s.q.shape, dtype=s.dt, device="cuda")
        k = torch.randn(s.T, 2, 128, device="cuda").bfloat16()
        rope = torch.randn(3300, 128, device="cuda")
        turned = torch.empty_like(q)
        s.cache.append(s.batch, 0, k, k, q=q, q_out=turned, rope=rope)
        s.cache.attend(s.batch, 0, turned, out, 0.1)
        torch.cuda.synchronize()
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=stream):
            s.cache.append(s.batch, 0, k, k, q=q, q_out=turned, rope=rope, stream=stream)
            s.cache.attend(s.batch, 0, turned, out, 0.1, stream=stream)
        for i in range(4):
            q.copy_(torch.randn(q.shape, device="cuda").bfloat16())
            k.copy_(torch.randn(k.shape, device="cuda").bfloat16())
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            s.cache.append(s.batch, 0, k, k, q=q, q_out=turned, rope=rope)
            s.cache.attend(s.batch, 0, turned, out, 0.1)
            torch.cuda.synchronize()
            assert torch.equal(got, out) and bool(torch.isfinite(out).all()), i
    finally:
        s.close()


def test_empty_batches():
    s = Setup([(10, 0), (0, 0)], 4, 2, 64)
    try:
        q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
        k = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
        s.cache.append(s.batch, 0, k, k)
        s.cache.attend(s.batch, 0, q, q, 1.0)
        none = s.cache.batch([], [0])
        s.cache.attend(none, 0, q, q, 1.0)
        torch.cuda.synchronize()
    finally:
        s.close()


def test_refusals():
    B, _K = _mods()
    s = Setup([(10, 1), (0, 20)], 4, 2, 64)
    try:
        q, h, st = s.q.cuda(), s.cache.handle, 0
        out = torch.full_like(q, 5.0)
        torch.cuda.synchronize()
        row = 4 * 64
        call = lambda batch=s.batch, layer=0, q_=q.data_ptr(), qs=row, o=out.data_ptr(), os_=row, scale=0.1: B.lora_kv_attend(h, batch, layer, q_, qs, o, os_, scale, st)  # noqa: E731
        for kw in (dict(layer=1), dict(layer=-1), dict(q_=0), dict(o=0), dict(q_=q.data_ptr() + 2), dict(o=out.data_ptr() + 8), dict(qs=row - 8), dict(os_=row + 1),
                   dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(batch=None), dict(o=q.data_ptr(), os_=2 * row)):
            assert call(**kw) == B.LORA_E_INVAL, kw
        assert B.lora_kv_attend(None, s.batch, 0, q.data_ptr(), row, out.data_ptr(), row, 0.1, st) == B.LORA_E_INVAL
        torch.cuda.synchronize()
        assert bool((out == 5).all())
        for t in (q[:5], q.float(), q.cpu(), q[..., :32], q.transpose(0, 1)):
            with pytest.raises(ValueError):
                s.cache.attend(s.batch, 0, t, out, 0.1)
        # a batch whose sequences were cut back, moved, ended or got a page of their own is of no use any more
        s.cache.fork(1, [2])
        assert call() == B.LORA_OK
        s.cache.extend([1], [1])
        assert call() == B.LORA_E_STATE
        s.cache.batch_destroy(s.batch)
        s.batch = s.cache.batch([0, 1], [0, 1, 1])
        s.cache.free([2])
        s.cache.truncate([1], [3])
        assert call(batch=s.batch) == B.LORA_E_STATE
        s.cache.batch_destroy(s.batch)
        assert call(batch=s.batch) == B.LORA_E_INVAL and B.lora_kv_batch_destroy(h, s.batch) == B.LORA_E_INVAL
        s.batch = s.cache.batch([0, 1], [0, 1, 2])
        s.cache.free([0])
        assert B.lora_kv_attend(h, s.batch, 0, q.data_ptr(), row, out.data_ptr(), row, 0.1, st) == B.LORA_E_STATE
    finally:
        s.close()
