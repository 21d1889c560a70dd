"""Pages of 8-bit values against their definition in 64 bits: what lora_kv_append stores, bit by bit; what lora_kv_seq_read gives back; attention over such
pages, at the lengths, heads and pages where it can go wrong."""
import math

import numpy as np
import pytest

import kv_e4m3_plain as plain
import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SEGS = [(0, 1), (7, 1), (15, 1), (16, 1), (0, 3), (5, 8), (0, 40), (61, 7), (64, 64), (31, 100), (10, 0), (0, 16), (3, 13)]


def _mods():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache
    return B, KvCache


def _cache(segs, heads, kv, dim, page, layers=1, **kw):
    _B, KvCache = _mods()
    need = sum(-(-(c + n) // page) for c, n in segs) + 3
    return KvCache(layers, heads, kv, dim, need, page_tokens=page, max_seqs=len(segs) + 1, max_batch_seqs=len(segs) + 1, max_batch_tokens=max(1, sum(n for _c, n in segs)), e4m3=True, **kw)


def _scatter(cache, segs, page):
    """The cached tokens of every sequence, page by page in turn: the pages of a sequence lie apart."""
    ids, ctx = np.arange(len(segs)), np.asarray([c for c, _n in segs])
    cache.add(ids)
    for at in range(0, int(ctx.max()), page):
        who = np.flatnonzero(ctx > at)
        cache.extend(who, np.minimum(page, ctx[who] - at))
    return np.concatenate([[0], np.cumsum([n for _c, n in segs])]).astype(np.int32)


def _sure(x, e):
    """Values that are not so near a border between two of 8 bits (2^-40 of themselves) that 64-bit arithmetic in another order may say otherwise."""
    y = np.abs(x) / 2.0 ** e[..., None].astype(np.float64)
    mid = (plain.MEANT[:126] + plain.MEANT[1:127]) / 2
    near = mid[np.clip(np.searchsorted(mid, y), 1, 125) + np.array([[-1], [0]]).reshape(2, *([1] * y.ndim))]
    return (np.abs(near - y) > 2.0**-40 * y).all(0) | ~np.isfinite(y)


def _append(segs, heads, kv, dim, page, rope_dim=None, neighbours=False, norm=False, strided=False, spread=0.0, layers=2, layer=1, plant=None, with_q=True):
    rope_dim = dim if rope_dim is None else rope_dim
    cache = _cache(segs, heads, kv, dim, page, layers)
    try:
        T = sum(n for _c, n in segs)
        gen = torch.Generator().manual_seed(5)
        host = torch.randint(0, 256, cache.pages.shape, generator=gen, dtype=torch.uint8)
        cache.pages.copy_(host)
        off = _scatter(cache, segs, page)
        batch = cache.batch(np.arange(len(segs)), off)
        wide = torch.randn(T, heads + 2 * kv + 1, dim, generator=gen) * torch.exp(spread * torch.randn(T, heads + 2 * kv + 1, 1, generator=gen))
        wide = wide.bfloat16()
        if plant is not None:
            plant(wide)
        q, k, v = wide[:, :heads], wide[:, heads : heads + kv], wide[:, heads + kv : heads + 2 * kv]
        pos = np.concatenate([np.arange(c, c + n) for c, n in segs])
        rope = torch.randn(int(pos.max()) + 1, rope_dim, generator=gen) if rope_dim else None
        weights = 1 + 0.5 * torch.randn(kv, dim, generator=gen) if norm else None
        dev = wide.cuda()
        qd, kd, vd = dev[:, :heads], dev[:, heads : heads + kv], dev[:, heads + kv : heads + 2 * kv]
        if not strided:
            qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
        q_out = torch.empty(T, heads, dim, device="cuda", dtype=torch.bfloat16)
        cache.append(batch, layer, kd, vd, q=qd if with_q else None, q_out=q_out if with_q else None, rope=None if rope is None else rope.cuda(), neighbours=neighbours,
                     k_norm=None if weights is None else weights.cuda(), eps=1e-5)
        torch.cuda.synchronize()
        with np.errstate(invalid="ignore"):
            want_k, want_v = k.double().numpy(), v.double().numpy()
            if norm:
                want_k = plain.norm(want_k, weights.numpy(), 1e-5)
            if rope_dim:
                want_k = kv_plain.turn(want_k, pos, rope.numpy(), neighbours)
        want, sure = host.numpy().copy(), np.ones(host.shape, bool)
        for x, key in ((want_k, True), (want_v, False)):
            e = plain.exponents(x)
            bits, certain = plain.to_bytes(x, e), np.ones(x.shape, bool)
            if key:  # what is neither normed nor turned is stored as it comes: there is no doubt about it
                made = dim if norm else rope_dim
                certain[..., :made] = _sure(x, e)[..., :made]
            for i, (c, n) in enumerate(segs):
                rows = slice(int(off[i]), int(off[i + 1]))
                for h in range(kv if n else 0):
                    where, keys, vals, ke, ve = (a[c:] for a in plain.places(cache.pages_of(i), page, dim, kv, h, c + n))
                    inner = keys if key else vals
                    want[where[:, None], layer, inner], sure[where[:, None], layer, inner] = bits[rows, h], certain[rows, h]
                    want[where, layer, ke if key else ve] = e[rows, h] + 127
        got = cache.pages.cpu().numpy()
        # (the sign of no number says nothing)
        differ = (got != want) & ~(((got & 127) == 127) & ((want & 127) == 127)) & sure
        assert not differ.any(), (np.argwhere(differ)[:5], got[differ][:5], want[differ][:5])
        assert sure.mean() > 0.999 or plant is not None
        # and read back, sequence by sequence in another order, as bf16 that are exactly what is stored
        ids = np.arange(len(segs))[::-1]
        n_all = np.asarray([sum(segs[i]) for i in ids])
        out = torch.zeros(2, int(n_all.sum()), kv + 1, dim, device="cuda", dtype=torch.bfloat16)
        cache.read(ids, layer, out[0, :, :kv], out[1, :, :kv])
        torch.cuda.synchronize()
        back, at = out.float().cpu().numpy(), 0
        assert not back[:, :, kv].any()
        for i, n in zip(ids, n_all):
            for h in range(kv if n else 0):
                with np.errstate(invalid="ignore", over="ignore"):
                    keys, vals = plain.read(got, cache.pages_of(int(i)), layer, h, kv, page, dim, int(n))
                    # exponents that were there before may be any: what bf16 can't hold is left out
                    for have, x in ((back[0, at : at + n, h], keys), (back[1, at : at + n, h], vals)):
                        own = np.arange(n) >= segs[i][0]
                        assert np.array_equal(have[own], x[own].astype(np.float32), equal_nan=True)
            at += n
        if with_q:
            return q_out.float().cpu().numpy(), q.float().numpy()
    finally:
        cache.close()


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dim,page,rope_dim", [(64, 32, 64), (128, 64, 128), (128, 128, 48), (256, 64, 256), (64, 256, 16), (64, 64, 0), (256, 32, 32)])
def test_what_is_stored(dim, page, rope_dim, neighbours):
    _append(SEGS, 6, 2, dim, page, rope_dim, neighbours, spread=1.0)
    _append(SEGS, 3, 3, dim, page, rope_dim, neighbours, spread=8.0, norm=True, strided=True)


def test_what_is_stored_by_large_batches_and_without_queries():
    _append([(0, 2900), (5, 77), (64, 1)], 42, 7, 64, 64, layers=1, layer=0)
    _append([(7, 1500)], 32, 16, 128, 128, 128, True, norm=True, layers=1, layer=0)
    _append(SEGS, 8, 1, 64, 32, with_q=False)


def test_largest_smallest_and_no_numbers():
    """Heads of zeros, of the smallest and largest values, of infinities and NaN beside others, of values on the borders."""
    def plant(wide):
        wide[0] = 0
        wide[1] = 2.0**-126
        wide[2] = 1.7e38
        wide[3, :, ::2], wide[3, :, 1::2] = 2.0**-100, 2.0**100
        wide[4, :, 3] = float("inf")
        wide[5, :, 3] = float("-inf")
        wide[6, :, 9] = float("nan")
        wide[7] = float("nan")
        wide[8] = 448.0
        wide[9, :, 0], wide[9, :, 1:] = 449.0, 1.0
        wide[10] = torch.arange(wide.shape[-1]) * 0.0625  # every other one half way between two of 8 bits
        wide[11] = (17 + 2 * torch.arange(wide.shape[-1]) % 16) / 16

    for dim in (64, 128):
        _append([(0, 12), (4, 24)], 2, 2, dim, 32, 0, plant=plant)
        _append([(4, 12)], 2, 2, dim, 32, 0, plant=plant)


def test_queries_are_those_of_bf16_pages():
    """Queries turn and are normed as they are beside pages of bf16, to the bit."""
    B, KvCache = _mods()
    x = torch.randn(50, 12, 64, device="cuda").bfloat16()
    rope, w = torch.randn(50, 64, device="cuda"), torch.rand(8, 64, device="cuda")
    outs = []
    for e4m3 in (False, True):
        cache = KvCache(1, 8, 2, 64, 4, page_tokens=64, max_seqs=1, max_batch_seqs=1, max_batch_tokens=50, e4m3=e4m3)
        cache.add([0])
        b = cache.batch([0], [0, 50])
        for q_norm in (None, w):
            outs.append(torch.empty(50, 8, 64, device="cuda", dtype=torch.bfloat16))
            cache.append(b, 0, x[:, 8:10], x[:, 10:], q=x[:, :8], q_out=outs[-1], rope=rope, q_norm=q_norm)
        cache.close()
    assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])


# ---- read back ------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page,kv", [(64, 32, 1), (128, 64, 3), (256, 128, 2), (64, 256, 5)])
def test_pages_of_every_type_are_read_back(dim, page, kv, dtype):
    B, KvCache = _mods()
    dt, u = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    lengths = [700, 1, 0, page, page + 1, 3 * page - 1]
    cache = KvCache(3, kv, kv, dim, 40 + 700 // page, page_tokens=page, max_seqs=8, max_batch_seqs=8, dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
    try:
        cache.add(np.arange(6))
        cache.extend(np.arange(6), lengths)
        cache.fork(0, [9], 650)
        gen = torch.Generator().manual_seed(1)
        host = torch.randn(cache.pages.shape, generator=gen).to(dt)
        cache.pages.copy_(host)
        pages = host.float().numpy()
        for ids, first, n in (([0, 1, 3, 4, 5, 9], None, None), ([5, 0, 0, 2, 9], [3, 650, 0, 0, 649], [2, 50, 1, 0, 1]), ([3], [page - 1], [1]), ([2], None, None)):
            counts = n or [cache.length(i) for i in ids]
            T = sum(counts)
            out = torch.full((T, 2 * kv + 1, dim), 7.0, device="cuda", dtype=dt)
            cache.read(ids, 2, out[:, kv : 2 * kv], out[:, :kv], first=first, n_tokens=n)
            torch.cuda.synchronize()
            got, at = out.float().cpu().numpy(), 0
            assert (got[:, 2 * kv] == 7).all()
            for i, f, m in zip(ids, first or [0] * len(ids), counts):
                for h in range(kv if m else 0):
                    k, v = kv_plain.read(pages, cache.pages_of(i), 2, h, page, dim, u, f + m)
                    assert np.array_equal(got[at : at + m, kv + h], k[f:]) and np.array_equal(got[at : at + m, h], v[f:])
                at += m
    finally:
        cache.close()


def test_more_pages_than_one_launch_reads():
    _B, KvCache = _mods()
    cache = KvCache(1, 1, 1, 64, 700, page_tokens=32, max_seqs=4, max_batch_seqs=4, e4m3=True)
    try:
        cache.add([0, 1])
        cache.extend([0, 1], [32 * 500 - 3, 40])
        gen = torch.Generator().manual_seed(1)
        host = torch.randint(0, 256, cache.pages.shape, generator=gen, dtype=torch.uint8)
        host[..., -64:] = torch.randint(100, 140, (700, 1, 64), generator=gen, dtype=torch.uint8)
        cache.pages.copy_(host)
        out = torch.empty(2, 32 * 500 + 37, 1, 64, device="cuda", dtype=torch.bfloat16)
        cache.read([1, 0], 0, out[0], out[1])
        got = out.float().cpu().numpy()
        for i, at, n in ((1, 0, 40), (0, 40, 32 * 500 - 3)):
            k, v = plain.read(host.numpy(), cache.pages_of(i), 0, 0, 1, 32, 64, n)
            assert np.array_equal(got[0, at : at + n, 0], k, equal_nan=True) and np.array_equal(got[1, at : at + n, 0], v, equal_nan=True)
    finally:
        cache.close()


def test_read_refusals():
    B, KvCache = _mods()
    cache = KvCache(2, 2, 2, 64, 8, page_tokens=32, max_seqs=3, max_batch_seqs=2, max_batch_tokens=40, e4m3=True)
    try:
        cache.add([0, 1])
        cache.extend([0], [30])
        out = torch.full((2, 30, 2, 64), 5.0, device="cuda", dtype=torch.bfloat16)
        p = out.data_ptr()
        good = dict(ids=[0], first=[0], n_tokens=[30], layer=0, k=p, k_stride=128, v=p + 30 * 256, v_stride=128, n_rows=30)
        for kw, rc in ((dict(ids=[7]), B.LORA_E_NOTFOUND), (dict(n_tokens=[31]), B.LORA_E_INVAL), (dict(first=[1]), B.LORA_E_INVAL), (dict(first=[-1]), B.LORA_E_INVAL),
                       (dict(n_tokens=[-1]), B.LORA_E_INVAL), (dict(ids=[1]), B.LORA_E_INVAL), (dict(layer=2), B.LORA_E_INVAL), (dict(layer=-1), B.LORA_E_INVAL), (dict(k=0), B.LORA_E_INVAL),
                       (dict(k=p + 2), B.LORA_E_INVAL), (dict(k_stride=120), B.LORA_E_INVAL), (dict(v_stride=132), B.LORA_E_INVAL), (dict(first=[2**31 - 1], n_tokens=[2**31 - 1]), B.LORA_E_INVAL),
                       (dict(n_rows=29), B.LORA_E_INVAL), (dict(n_rows=31), B.LORA_E_INVAL), (dict(n_rows=-1), B.LORA_E_INVAL), (dict(n_rows=2**33), B.LORA_E_INVAL), (dict(n_tokens=None, first=[1]), B.LORA_E_INVAL)):
            assert B.lora_kv_seq_read(cache.handle, **{**good, **kw}) == rc, kw
        for kw in (dict(v=out[1, :29]), dict(k=out[0].float()), dict(v=out[1, :, :1])):
            with pytest.raises(ValueError):
                cache.read([0], 0, **{**dict(k=out[0], v=out[1]), **kw})
        with pytest.raises(B.LoraError):
            cache.read([0], 0, out[0, :29], out[1, :29])
        torch.cuda.synchronize()
        assert bool((out == 5).all())
        assert B.lora_kv_seq_read(cache.handle, [], [], [], 0, 0, 0, 0, 0, 0) == 0 and B.lora_kv_seq_read(cache.handle, [1], None, None, 0, 0, 0, 0, 0, 0) == 0
        with pytest.raises(ValueError):
            KvCache(1, 2, 2, 64, 8, e4m3=True, pages=torch.empty(8, 1, 2 * 2 * 64 * 65, device="cuda", dtype=torch.int8))
    finally:
        cache.close()


# ---- attention --------------------------------------------------------------------------------------

class Setup:
    """Sequences with scattered pages of 8-bit values and a batch: segs is [(cached tokens, new tokens)]."""

    def __init__(self, segs, heads, kv, dim, page=64, seed=0, layers=1, exps=(118, 124), beyond=None):
        self.segs, self.heads, self.kv, self.dim, self.page, self.layers = segs, heads, kv, dim, page, layers
        self.cache = _cache(segs, heads, kv, dim, page, layers)
        self.offsets = _scatter(self.cache, segs, page)
        self.batch = self.cache.batch(np.arange(len(segs)), self.offsets)
        self.tables = [self.cache.pages_of(i) for i in range(len(segs))]
        gen = torch.Generator().manual_seed(seed)
        # values as append stores them: the token's largest between 224 and 448
        split = 2 * kv * page * dim
        x = (torch.randn(*self.cache.pages.shape[:2], split, generator=gen) * 100).clamp(-448, 448)
        self.host = torch.empty(self.cache.pages.shape, dtype=torch.uint8)
        self.host[..., :split] = x.to(torch.float8_e4m3fn).view(torch.uint8)
        self.host[..., split:] = torch.randint(*exps, self.host[..., split:].shape, generator=gen, dtype=torch.uint8)
        if beyond is not None:  # every byte that no sequence holds
            a, b = np.full(self.host.shape, beyond, np.uint8), self.host.numpy()
            for i, (c, n) in enumerate(segs):
                for h in range(kv if c + n else 0):
                    where, keys, vals, ke, ve = plain.places(self.tables[i], page, dim, kv, h, c + n)
                    for inner in (keys, vals):
                        a[where[:, None], :, inner] = b[where[:, None], :, inner]
                    for inner in (ke, ve):
                        a[where, :, inner] = b[where, :, inner]
            self.host = torch.from_numpy(a)
        self.cache.pages.copy_(self.host)
        self.T = int(self.offsets[-1])
        self.q = torch.randn(self.T, heads, dim, generator=gen).bfloat16()

    def check(self, scale=None, layer=0, q=None, batch=None):
        scale = 1.0 / math.sqrt(self.dim) if scale is None else scale
        qd = (self.q if q is None else q).cuda()
        out = torch.full(qd.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        self.cache.attend(self.batch if batch is None else batch, layer, qd, out, scale)
        torch.cuda.synchronize()
        got, pages, q = out.float().cpu().numpy(), self.host.numpy(), qd.float().cpu().numpy()
        eps, longest = 2.0**-24, max(c + n for c, n in self.segs)
        for i, (c, n) in enumerate(self.segs):
            rows = slice(int(self.offsets[i]), int(self.offsets[i + 1]))
            for g in range(self.kv if n else 0):
                k, v = plain.read(pages, self.tables[i], layer, g, self.kv, self.page, self.dim, c + n)
                for h in range(g * (self.heads // self.kv), (g + 1) * (self.heads // self.kv)):
                    want, mass, reach = kv_plain.attend(q[rows, h], k, v, c, scale)
                    # the keys and values are exact in bf16, so what rounding can do is what it can over pages of bf16: a score is off by dim products' roundings, every weight
                    # by 2^-8 of itself, and the output by half a step
                    bound = mass * ((2 * self.dim + 8) * eps * reach[..., None] + (longest + 16) * 2 * eps) + 2.0**-8 * mass + 2.0**-8 * (np.abs(want) + 2.0**-7 * mass) + 1e-38
                    over = np.abs(got[rows, h] - want) - bound
                    assert np.isfinite(got[rows, h]).all() and (over <= 0).all(), (self.segs[i], h, np.unravel_index(np.argmax(over), over.shape), float(over.max()))
        return out

    def close(self):
        self.cache.close()


def _check(segs, heads, kv, dim, **kw):
    scale, layer = kw.pop("scale", None), kw.pop("layer", 0)
    s = Setup(segs, heads, kv, dim, **kw)
    try:
        s.check(scale, layer)
    finally:
        s.close()


TOKENS = [(0, 1), (1, 1), (15, 1), (16, 1), (30, 1), (31, 1), (32, 1), (63, 1), (64, 1), (127, 1), (130, 1), (255, 1), (256, 1), (700, 1)]
PROMPTS = [(0, 1), (0, 3), (0, 33), (5, 29), (31, 32), (64, 64), (0, 127), (1, 128), (127, 130), (300, 17), (0, 0), (90, 0)]


@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64), (128, 32), (256, 32), (128, 256), (64, 128), (256, 64)])
@pytest.mark.parametrize("heads,kv", [(4, 4), (6, 2), (5, 1)])
def test_tokens_and_prompts(heads, kv, dim, page):
    _check(TOKENS, heads, kv, dim, page=page, seed=1)
    _check(PROMPTS, heads, kv, dim, page=page, seed=2)


@pytest.mark.parametrize("heads,kv,dim", [(16, 2, 128), (17, 1, 64), (32, 1, 128), (20, 4, 64), (130, 1, 64), (8, 8, 64), (7, 7, 128)])
def test_groups_of_every_kind(heads, kv, dim):
    _check([(45, 1), (0, 1), (63, 2), (99, 3), (0, 9), (10, 16), (200, 1)], heads, kv, dim, page=32, seed=3)


@pytest.mark.parametrize("segs,heads,kv,dim", [
    ([(9001, 1)], 8, 1, 128), ([(4999, 1), (0, 1), (3333, 1)], 4, 2, 64), ([(6000, 5)], 2, 2, 128), ([(5000, 40)], 8, 2, 64),
    ([(3000, 200), (12, 1), (2500, 1)], 4, 1, 128), ([(4100, 33)], 2, 1, 256), ([(2047, 1), (2048, 1), (2049, 1)], 40, 8, 64)])
def test_long_caches_are_cut_and_joined(segs, heads, kv, dim):
    s = Setup(segs, heads, kv, dim, seed=4)
    try:
        assert _mods()[0].lora_kv_batch_info(s.batch)[1].n_joins > 0
        s.check()
    finally:
        s.close()


def test_few_blocks_are_even():
    """Pieces are made a little longer where the blocks would be a few more than the compute units take at a time, and outputs are right for all that."""
    B, _K = _mods()
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    for segs, heads, kv, dim in (([(16000, 1)] * 4, 16, 8, 64), ([(3000, 40), (2000, 8)], 8, 4, 128), ([(1500, 1)] * 20, 8, 8, 64), ([(4000, 64)], 8, 2, 256)):
        s = Setup(segs, heads, kv, dim, seed=11)
        try:
            rc, info = B.lora_kv_batch_info(s.batch)
            blocks = (info.n_row_items + info.n_tile_items) * kv
            assert rc == 0 and (blocks <= 2 * n_cu or n_cu < 256), (segs[0], blocks)
            s.check()
        finally:
            s.close()


def test_batches_of_many_requests():
    _check([(20 + i % 90, 1) for i in range(300)], 8, 8, 64, page=32, seed=5)
    _check([(i % 50, 1 + i % 40) for i in range(60)], 8, 2, 128, seed=6, layers=2, layer=1)


@pytest.mark.parametrize("byte", [255, 127, 0])
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64), (256, 128)])
def test_what_no_sequence_holds_is_never_used(dim, page, byte):
    """Every other byte of the pages is no number, exponents that are none among them."""
    _check(TOKENS, 4, 2, dim, page=page, seed=7, beyond=byte)
    _check(PROMPTS, 4, 2, dim, page=page, seed=8, beyond=byte)
    _check([(2500, 1), (700, 200)], 8, 1, dim, page=page, seed=9, beyond=byte)


@pytest.mark.parametrize("dim", [64, 128])
def test_hidden_tokens_that_are_no_numbers(dim):
    """A key or value beyond a token's position has no influence, whatever it is; one that a token sees and that is no number makes its outputs none."""
    s = Setup([(40, 100), (30, 1)], 4, 2, dim, seed=10)
    try:
        clean = s.check()
        for h in range(2):
            where, keys, vals, _ke, _ve = plain.places(s.tables[0], s.page, dim, 2, h, 140)
            for inner in (keys, vals):
                s.cache.pages[int(where[100]), 0, torch.from_numpy(inner[100]).cuda()] = 127
        out = torch.empty_like(clean)
        s.cache.attend(s.batch, 0, s.q.cuda(), out, 1.0 / math.sqrt(dim))
        torch.cuda.synchronize()
        assert torch.isfinite(out[:60]).all() and torch.isnan(out[60:100]).all() and torch.equal(out[100], clean[100])
        # (the rows before it are worked out in another order)
        assert float((out[:60].float() - clean[:60].float()).abs().max()) <= 2.0**-7 * float(clean[:60].float().abs().max())
    finally:
        s.close()


def test_exponents_from_end_to_end():
    """Scores and outputs with the smallest and the largest exponents that append stores."""
    _check([(90, 1), (0, 50)], 4, 2, 64, seed=11, exps=(10, 14))
    s = Setup([(90, 1), (0, 50)], 4, 2, 64, seed=12, exps=(240, 244))
    try:
        s.q = s.q * 2.0**-120  # scores of an ordinary size
        s.check()
    finally:
        s.close()


@pytest.mark.parametrize("page", [32, 64])
def test_large_tiles(page):
    """Prompts long enough for tiles of 256 rows, in pages of less than their stages' 64 tokens too: the last rows of some heads, whose lengths end inside everything."""
    B, _K = _mods()
    segs, heads, kv, dim = [(0, 2500), (700, 1700), (0, 2111)], 64, 8, 128
    s = Setup(segs, heads, kv, dim, page=page, seed=13)
    try:
        assert B.lora_kv_batch_info(s.batch)[1].tiles_way == B.LORA_KV_TILES_TURNS
        out = torch.full(s.q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
        s.cache.attend(s.batch, 0, s.q.cuda(), out, 1.0 / math.sqrt(dim))
        torch.cuda.synchronize()
        got, q, pages = out.float().cpu().numpy(), s.q.float().numpy(), s.host.numpy()
        assert np.isfinite(got).all()
        for i, (c, n) in enumerate(segs):
            for h in (0, 13, 63):
                k, v = plain.read(pages, s.tables[i], 0, h // 8, kv, page, dim, c + n)
                for t in (0, 1, 31, 32, 63, 100, n - 33, n - 2, n - 1):
                    at = int(s.offsets[i]) + t
                    want, mass, _r = kv_plain.attend(q[at : at + 1, h], k[: c + t + 1], v[: c + t + 1], c + t, 1.0 / math.sqrt(dim))
                    # every weight is off by 2^-8 of itself, the output by half a step; what fp32 loses is 2^-12 at these lengths
                    assert (np.abs(got[at, h] - want[0]) <= (2.0**-7 + 2.0**-12) * mass[0]).all(), (i, h, t)
    finally:
        s.close()


@pytest.mark.parametrize("segs,heads,kv", [([(0, 700)], 32, 32), ([(0, 700), (333, 1)], 32, 8), ([(300, 333), (0, 5)], 16, 4), ([(0, 1), (0, 129)], 8, 2)])
@pytest.mark.parametrize("page", [32, 128])
def test_heads_of_64_with_two_groups_to_a_tile(segs, heads, kv, page):
    B, _K = _mods()
    s = Setup(segs, heads, kv, 64, page=page, seed=14)
    try:
        assert B.lora_kv_batch_info(s.batch)[1].tiles_way == B.LORA_KV_TILES_PAIRS
        s.check()
    finally:
        s.close()


# ---- streams, graphs, large caches --------------------------------------------------------------------

def test_append_attend_and_read_captured_together():
    """A graph of an append, attention and a read gives an eager run's bits at every replay, with eager work of the same cache between the replays."""
    segs = [(100, 1), (0, 40), (33, 2)]
    cache = _cache(segs, 8, 2, 64, 32)
    try:
        off = _scatter(cache, segs, 32)
        cache.pages.random_(0, 120)
        cache.pages[..., -2 * 2 * 32 :].fill_(120)
        batch, T = cache.batch(np.arange(3), off), int(off[-1])
        x, rope = torch.randn(T, 12, 64, device="cuda").bfloat16(), torch.randn(200, 64, device="cuda").clamp(-1, 1)
        q, out = (torch.empty(T, 8, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        back = torch.empty(2, sum(c + n for c, n in segs), 2, 64, device="cuda", dtype=torch.bfloat16)

        def run(stream=None):
            cache.append(batch, 0, x[:, 8:10], x[:, 10:], q=x[:, :8], q_out=q, rope=rope, stream=stream)
            cache.attend(batch, 0, q, out, 0.125, stream=stream)
            cache.read([2, 0, 1], 0, back[0], back[1], stream=stream)

        run()
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            run(side)
        for i in range(4):
            x.copy_(torch.randn(x.shape, device="cuda"))
            run()
            torch.cuda.synchronize()
            want = [t.clone() for t in (q, out, back, cache.pages)]
            for t in (q, out, back):
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (q, out, back, cache.pages))), i
    finally:
        cache.close()


def test_reads_follow_appends_on_other_streams():
    _B, KvCache = _mods()
    cache = KvCache(1, 2, 2, 128, 70, page_tokens=64, max_seqs=2, max_batch_seqs=2, max_batch_tokens=4096, e4m3=True)
    try:
        cache.add([0])
        b = cache.batch([0], [0, 4000])
        big = torch.randn(4096, 4096, device="cuda")
        one, two = torch.cuda.Stream(), torch.cuda.Stream()
        back = torch.zeros(2, 4000, 2, 128, device="cuda", dtype=torch.bfloat16)
        for i in range(5):
            torch.cuda.synchronize()
            with torch.cuda.stream(one):
                k = torch.zeros(4000, 2, 128, device="cuda", dtype=torch.bfloat16)
                for _ in range(3):
                    big = big @ big * 1e-3
                k.fill_(float(2**i))
                cache.append(b, 0, k, k, stream=one)
            with torch.cuda.stream(two):
                cache.read([0], 0, back[0], back[1], stream=two)
            torch.cuda.synchronize()
            assert bool((back == 2**i).all()), i
    finally:
        cache.close()


def test_pages_beyond_4_gb():
    """Pages whose bytes lie beyond what 32 bits name: stored, attended to, read back."""
    _B, KvCache = _mods()
    kv, dim, page, n_pages = 32, 128, 64, 9000
    cache = KvCache(1, kv, kv, dim, n_pages, page_tokens=page, max_seqs=2, max_batch_seqs=2, max_batch_tokens=200, e4m3=True)
    try:
        assert cache.pages.numel() > 1 << 32
        cache.add([0, 1])
        cache.extend([0], [(n_pages - 4) * page])
        b = cache.batch([1], [0, 150])
        assert cache.pages_of(1).min() >= n_pages - 4
        x = torch.randn(150, 3 * kv, dim, device="cuda").bfloat16()
        cache.append(b, 0, x[:, kv : 2 * kv], x[:, 2 * kv :])
        out, back = torch.empty(150, kv, dim, device="cuda", dtype=torch.bfloat16), torch.empty(2, 150, kv, dim, device="cuda", dtype=torch.bfloat16)
        cache.attend(b, 0, x[:, :kv], out, dim**-0.5)
        cache.read([1], 0, back[0], back[1])
        torch.cuda.synchronize()
        k, v = x[:, kv : 2 * kv].double().cpu().numpy(), x[:, 2 * kv :].double().cpu().numpy()
        for have, want in ((back[0], k), (back[1], v)):
            e = plain.exponents(want)
            assert np.array_equal(have.double().cpu().numpy(), plain.MEANT[plain.to_bytes(want, e)] * 2.0 ** e[..., None])
        k, v, got, q = back[0].float().cpu().numpy(), back[1].float().cpu().numpy(), out.float().cpu().numpy(), x[:, :kv].float().cpu().numpy()
        for h in (0, 17, 31):
            want, mass, _r = kv_plain.attend(q[:, h], k[:, h], v[:, h], 0, dim**-0.5)
            assert (np.abs(got[:, h] - want) <= (2.0**-7 + 2.0**-12) * mass).all()
    finally:
        cache.close()
