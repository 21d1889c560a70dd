"""lora_kv_append_norm against its definition in 64 bits: norms of every head of queries and keys before they turn, in one pass."""
import numpy as np
import pytest

import kv_e4m3_plain
import kv_plain

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

SEGS = [(0, 1), (7, 1), (8, 1), (0, 3), (5, 8), (0, 40), (61, 7), (64, 64), (31, 100), (10, 0), (0, 16)]
EPS = 1e-5


def _mods():
    from paper_2411_17741_amd import binding as B
    from paper_2411_17741_amd.kv import KvCache
    return B, KvCache


def _run(segs, heads, kv, dim, page, dtype, rope_dim=None, neighbours=False, which="qk", per_head=False, strided=False, size=1.0, layers=2, layer=1):
    B, KvCache = _mods()
    dt, u = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    rope_dim = dim if rope_dim is None else rope_dim
    T = sum(n for _c, n in segs)
    cache = KvCache(layers, heads, kv, dim, sum(-(-(c + n) // page) for c, n in segs) + 2, page_tokens=page, max_seqs=len(segs), max_batch_seqs=len(segs),
                    max_batch_tokens=T, dtype=B.LORA_BF16 if dtype == "bf16" else B.LORA_F32)
    try:
        gen = torch.Generator().manual_seed(3)
        host = torch.randn(cache.pages.shape, generator=gen).to(dt)
        cache.pages.copy_(host)
        ids = np.arange(len(segs))
        cache.add(ids)
        cache.extend(ids, [c for c, _n in segs])
        off = np.concatenate([[0], np.cumsum([n for _c, n in segs])]).astype(np.int32)
        batch = cache.batch(ids, off)
        wide = (size * torch.randn(T, heads + 2 * kv + 1, dim, generator=gen)).to(dt)
        q, k, v = wide[:, :heads], wide[:, heads : heads + kv], wide[:, heads + kv : heads + 2 * kv]
        pos = np.concatenate([np.arange(c, c + n) for c, n in segs])
        rope = torch.randn(int(pos.max()) + 1, rope_dim, generator=gen) if rope_dim else None
        weights = lambda n: 1 + 0.5 * torch.randn(*((n, dim) if per_head else (dim,)), generator=gen)  # noqa: E731
        q_norm, k_norm = (weights(heads) if "q" in which else None), (weights(kv) if "k" in which else None)
        dev = wide.cuda()
        qd, kd, vd = dev[:, :heads], dev[:, heads : heads + kv], dev[:, heads + kv : heads + 2 * kv]
        if not strided:
            qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
        on = lambda t: None if t is None else t.cuda()  # noqa: E731
        kw = dict(rope=on(rope), neighbours=neighbours, q_norm=on(q_norm), k_norm=on(k_norm), eps=EPS)
        q_out = torch.full((T, heads + 1, dim), 3.0, dtype=dt, device="cuda")
        cache.append(batch, layer, kd, vd, q=qd, q_out=q_out[:, :heads], **kw)
        torch.cuda.synchronize()
        f = lambda t: t.float().numpy().astype(np.float64)  # noqa: E731

        def want(x, w):
            """-> the outputs, and what roundings can do to them.  In fp32 the factor is rounded, its product with the weight, and that with the value: 3 * 2^-24 of each normed
            value; two products and their sum make 2 more of each term (or 1, fused).  The squares of bf16 values are summed in fp32: two roundings for each of 8 pairs and one for each
            of up to 5 exchanges, 21 * 2^-24 of the sum, half of that in its root, and 2 for the quotient, the sum with eps and the root's own ulp (which is 2 * 2^-24): 14 more.  Then the
            output is rounded, by half a step."""
            x = f(x) if w is None else kv_e4m3_plain.norm(f(x), w.numpy(), EPS)
            y, terms = (kv_plain.turn(x, pos, rope.numpy(), neighbours), None) if rope_dim else (x, None)
            if rope_dim:  # the sum of the terms' sizes: turned with every sign such that nothing cancels
                r = np.abs(rope.numpy())
                terms = np.maximum(np.abs(kv_plain.turn(np.abs(x), pos, r, neighbours)), np.abs(kv_plain.turn(np.abs(x), pos, np.concatenate([r[:, : rope_dim // 2], -r[:, rope_dim // 2 :]], 1), neighbours)))
            else:
                terms = np.abs(x)
            e = (5 if dtype == "f32" or w is None else 19) * 2.0**-24 * terms
            half = 2.0**-8 if dtype == "bf16" else 2.0**-24
            e = e + half * (np.abs(y) + e)
            if w is None:
                e[..., rope_dim:] = 0  # neither normed nor turned: the same bits
            return y, e

        want_pages = host.float().numpy().astype(np.float64)
        slack = np.zeros(want_pages.shape)
        want_k, off_k = want(k, k_norm)
        for i, (c, n) in enumerate(segs):
            table, rows = cache.pages_of(i), slice(int(off[i]), int(off[i + 1]))
            for h in range(kv if n else 0):
                kv_plain.write(want_pages, table, layer, h, page, dim, u, c, want_k[rows, h], f(v)[rows, h])
                kv_plain.write(slack, table, layer, h, page, dim, u, c, off_k[rows, h], 0.0)
        got = cache.pages.float().cpu().numpy()
        assert (np.abs(got - want_pages) <= slack).all()
        want_q, off_q = want(q, q_norm)
        got_q = q_out.float().cpu().numpy()
        assert (np.abs(got_q[:, :heads] - want_q) <= off_q).all() and (got_q[:, heads] == 3).all()
        if not strided:  # in place
            cache.append(batch, layer, kd, vd, q=qd, **kw)
            assert torch.equal(qd, q_out[:, :heads])
        assert torch.equal(cache.pages.cpu(), torch.from_numpy(got).to(dt))
    finally:
        cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dim,page,rope_dim", [(64, 32, 64), (128, 64, 128), (128, 128, 48), (256, 64, 256), (64, 256, 16), (64, 64, 0), (256, 32, 32)])
def test_norms_before_turns(dim, page, rope_dim, neighbours, dtype):
    _run(SEGS, 6, 2, dim, page, dtype, rope_dim, neighbours)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["q", "k", "qk"])
@pytest.mark.parametrize("per_head", [False, True])
def test_weights_of_every_kind(which, per_head, dtype):
    _run(SEGS, 5, 5, 128, 64, dtype, which=which, per_head=per_head, strided=True)
    _run([(999, 1)], 1, 1, 64, 64, dtype, which=which, per_head=per_head)
    _run([(3, 2)], 7, 1, 256, 32, dtype, 64, which=which, per_head=per_head)


@pytest.mark.parametrize("neighbours", [False, True])
def test_large_batches(neighbours):
    """Beyond the size from which a thread takes more heads, in numbers of heads that its share does not divide."""
    _run([(0, 2900), (5, 77), (64, 1)], 42, 7, 64, 64, "bf16", 64, neighbours, layers=1, layer=0)
    _run([(3, 2990)], 40, 4, 64, 32, "f32", 32, neighbours, strided=True, per_head=True, layers=1, layer=0)


@pytest.mark.parametrize("size", [1e-18, 1e18])
def test_values_whose_squares_leave_fp32(size):
    """Values of 1e18 times a few have squares of 1e37 and their sum is beyond fp32's range; those of 1e-18 count for little beside eps."""
    _run([(0, 33), (70, 1)], 4, 2, 128, 64, "bf16", size=size)
    _run([(0, 33), (70, 1)], 4, 2, 128, 64, "f32", size=size)


@pytest.mark.parametrize("size", [1e-19, 4e-19, 1e-16])
def test_values_whose_squares_are_below_the_normal_numbers(size, monkeypatch):
    """... with the smallest eps there is, beside which they count."""
    monkeypatch.setitem(globals(), "EPS", 2.0**-126)
    for dtype in ("bf16", "f32"):
        _run([(0, 33), (70, 1)], 4, 2, 128, 64, dtype, size=size)


def test_heads_of_zeros_and_of_no_numbers():
    """A head of zeros stays one; a NaN spoils its own head and nothing else."""
    _B, KvCache = _mods()
    cache = KvCache(1, 2, 2, 64, 4, page_tokens=32, max_seqs=2, max_batch_seqs=2, max_batch_tokens=40)
    try:
        cache.pages.zero_()
        cache.add([0])
        b = cache.batch([0], [0, 20])
        k = torch.ones(20, 2, 64, device="cuda").bfloat16()
        k[3, 1], k[7, 0, 5] = 0, float("nan")
        w = torch.full((64,), 2.0, device="cuda")
        q = k.clone()
        cache.append(b, 0, k, k, q=q, q_norm=w, k_norm=w)
        got = cache.pages[0].float().cpu().numpy()[None]
        for h in range(2):
            keys, vals = kv_plain.read(got, [0], 0, h, 32, 64, 8, 20)
            bad = np.zeros((20, 64), bool)
            bad[7] = h == 0
            assert np.array_equal(np.isnan(keys), bad) and np.array_equal(vals, k[:, h].float().cpu().numpy(), equal_nan=True)
            assert np.array_equal(q[:, h].float().cpu().numpy(), keys, equal_nan=True)
            sure = np.full((20, 64), 2.0)
            sure[3] = 0 if h == 1 else 2
            assert (keys[~bad] == sure[~bad]).all()
    finally:
        cache.close()


def test_captured_and_replayed():
    """A captured append with norms gives an eager one's bits at every replay, with eager work between the replays."""
    _B, KvCache = _mods()
    cache = KvCache(1, 8, 2, 128, 8, page_tokens=64, max_seqs=2, max_batch_seqs=2, max_batch_tokens=100)
    try:
        cache.pages.zero_()
        cache.add([0, 1])
        b = cache.batch([0, 1], [0, 77, 78])
        x = torch.randn(78, 12, 128, device="cuda").bfloat16()
        w, rope = torch.rand(128, device="cuda"), torch.randn(80, 128, device="cuda")
        out = torch.empty(78, 8, 128, device="cuda", dtype=torch.bfloat16)
        call = lambda stream=None: cache.append(b, 0, x[:, 8:10], x[:, 10:], q=x[:, :8], q_out=out, rope=rope, q_norm=w, k_norm=w, stream=stream)  # noqa: E731
        call()
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            call(side)
        for i in range(3):
            x.copy_(torch.randn(x.shape, device="cuda"))
            call()
            torch.cuda.synchronize()
            want, pages = out.clone(), cache.pages.clone()
            out.zero_(), cache.pages.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(cache.pages, pages), i
    finally:
        cache.close()


def test_refusals():
    B, KvCache = _mods()
    cache = KvCache(2, 4, 2, 64, 8, page_tokens=32, max_seqs=2, max_batch_seqs=2, max_batch_tokens=40)
    try:
        cache.pages.zero_()
        cache.add([0])
        b = cache.batch([0], [0, 5])
        k = torch.ones(5, 2, 64, device="cuda").bfloat16()
        q = torch.ones(5, 4, 64, device="cuda").bfloat16()
        w = torch.ones(4, 68, device="cuda")
        torch.cuda.synchronize()
        kp, qp, wp = k.data_ptr(), q.data_ptr(), w.data_ptr()
        good = dict(layer=0, k=kp, v=kp, k_stride=128, v_stride=128, q=qp, q_out=qp, q_stride=256, q_out_stride=256, q_norm=wp, k_norm=wp, q_norm_stride=68)
        no_q = dict(q=0, q_out=0, q_stride=0, q_out_stride=0)
        for kw in (dict(layer=2), dict(k=0), dict(q_norm=wp + 4), dict(k_norm=wp + 8), dict(q_norm_stride=60), dict(q_norm_stride=66), dict(k_norm_stride=-64), dict(eps=0.0),
                   dict(eps=-1e-6), dict(eps=1e-39), dict(eps=float("inf")), dict(eps=float("nan")), no_q):
            assert B.lora_kv_append_norm(cache.handle, b, **{**good, **kw}) == B.LORA_E_INVAL, kw
        torch.cuda.synchronize()
        assert not cache.pages.any() and bool((q == 1).all())
        assert B.lora_kv_append_norm(cache.handle, b, **good) == B.LORA_OK
        assert B.lora_kv_append_norm(cache.handle, b, **{**good, **no_q, "q_norm": 0}) == B.LORA_OK
        for kw in (dict(q_norm=w[0, :64]), dict(q=q, q_norm=w[0]), dict(q=q, q_norm=w[:, :64].half()), dict(k_norm=w[:, :64]), dict(k_norm=w[:2, :64].cpu()), dict(q=q, q_norm=w[:1, :64]),
                   dict(q=q, q_norm=w.t()[:64].t().contiguous().t().contiguous().t())):
            with pytest.raises(ValueError):
                cache.append(b, 0, k, k, **kw)
        cache.append(b, 0, k, k, q=q, q_norm=w[:, :64], k_norm=w[0, :64])
        cache.truncate([0], [1])
        assert B.lora_kv_append_norm(cache.handle, b, **good) == B.LORA_E_STATE
        torch.cuda.synchronize()
    finally:
        cache.close()
